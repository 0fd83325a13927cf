"""Log probabilities of given tokens, entropies, alternatives and their gradient against plain forms in 64 bits.

Tolerances.  With tau the temperature, m a row's largest logit and d = (m - x) / tau log2(e) >= 0 the kernels work out 2^(x c - R), c = log2(e) / tau
rounded once: relative to the largest word's that is off by 2^-22 (the exponential) and 2^-23 d (c, and the rounding of x c - R, which is less
than d + 1), so by 2^-22 (2 + d).  Sums of such terms in single precision add `DEPTH` 2^-24.  All of it falls on the words below the largest only:
with `rest` their share, log Z is off by delta rest, and so is the mean of d by delta (mean + 2 rest) with twice that delta (terms
of the size e (d + 1), of which e d is wanted).  What comes out is rounded once.
"""
import math

import pytest
import torch

from paper_1412_1576_b200 import binding as b
from paper_1412_1576_b200 import cache, rows

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF_STEP = {F32: 2.0**-24, F16: 2.0**-11, BF16: 2.0**-8}
SMALLEST = {F32: 2.0**-150, F16: 2.0**-25, BF16: 2.0**-134}
DEPTH = 160
NAN, INF = float("nan"), float("inf")


def make(n, V, dtype, seed, pad=0, spread=3.0, offset=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, V, generator=g) * spread).to(dtype)
    flat = torch.full((offset + n * (V + pad),), 77.0, dtype=dtype, device="cuda")
    view = flat[offset:].view(n, V + pad)[:, :V]
    view.copy_(x)
    tokens = torch.randint(0, V, (n,), generator=g).to(torch.int32)
    return view, tokens.cuda()


def reference(x, tokens, tau):
    """x in 64 bits: log q, logprobs and entropy with their bounds, and what the gradient's bound needs."""
    x = x.double()
    n, V = x.shape
    m = x.max(1, keepdim=True).values
    log_q = torch.log_softmax(x / tau, 1)
    q = torch.exp(log_q)
    d = torch.nan_to_num((m - x) / tau, nan=0.0, posinf=0.0)
    below = torch.where(x < m, q, 0.0)
    rest, mean = below.sum(1), (below * d).sum(1)
    log2 = 1.4427 * torch.where(rest > 0, mean / rest, 0.0)           # mean of d over the words below the largest
    delta = 2.0**-22 * (2 + log2) + DEPTH * 2.0**-24
    known = (tokens >= 0) & (tokens < V)
    at = torch.where(known, tokens, 0).long()[:, None]
    # where the largest word is nearly sure the logarithm of its share is that of one minus the rest
    sure = torch.log1p(-rest) - torch.log((x == m).sum(1).double())
    lp = torch.where((torch.gather(x, 1, at) == m)[:, 0], sure, torch.gather(log_q, 1, at)[:, 0])
    lp = torch.where(known, lp, 0.0)
    entropy = torch.where(q > 0, -q * torch.where(x == m, sure[:, None], log_q), 0.0).sum(1)
    lp_tol = torch.where(known, delta * rest, 0.0) + HALF_STEP[F32] * lp.abs() + 2.0**-149
    entropy_tol = delta * rest + 2 * delta * (mean + 2 * rest) + HALF_STEP[F32] * entropy.abs() + 2.0**-149
    return log_q, lp, lp_tol, entropy, entropy_tol


def close(got, want, tol):
    got, want, tol = got.cpu().double(), want.cpu(), tol.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    plain = torch.isfinite(want)
    assert torch.equal(got[~plain & ~torch.isnan(want)], want[~plain & ~torch.isnan(want)])
    off = (got - want).abs()
    assert bool((off <= tol)[plain].all()), float((off / tol)[plain].max())


def check(x, tokens, top=0, tau=1.0):
    got = rows.token_logprobs(x, tokens, top=top, temperature=tau)
    log_q, lp, lp_tol, entropy, entropy_tol = reference(x, tokens, tau)
    close(got.logprobs, lp, lp_tol)
    close(got.entropy, entropy, entropy_tol)
    assert (got.ids is None) == (got.alternatives is None) == (top == 0)
    if top:
        ids, _, _ = rows.top_logits(x, top, temperature=tau)
        assert torch.equal(got.ids, ids)
        there = ids >= 0
        want = torch.gather(log_q, 1, ids.long().clamp(min=0))
        # (the bound of a log probability: that of log Z, whichever word it is; a likely one's own by its complement)
        best = (torch.gather(x.double(), 1, ids.long().clamp(min=0)) == x.double().max(1, keepdim=True).values) & there
        first = reference(x, x.double().argmax(1).to(torch.int32), tau)
        want = torch.where(best, first[1][:, None], want)
        close(got.alternatives, torch.where(there, want, -INF), (lp_tol + first[2])[:, None] + HALF_STEP[F32] * want.abs())
    # the same call, the same bits
    again = rows.token_logprobs(x, tokens, top=top, temperature=tau)
    assert all(torch.equal(a.nan_to_num(5.0), c.nan_to_num(5.0)) for a, c in zip(got, again) if a is not None)
    return got


SIZES = [(1, 1), (3, 1), (5, 2), (2, 7), (4, 31), (3, 32), (7, 255), (3, 256), (2, 1000), (1, 4099), (9, 10_000), (300, 2_049), (2, 50_021),
         (3, 131_072), (2, 141_000), (1, 1 << 20), (600, 3001)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,V", SIZES)
def test_logprobs(n, V, dtype):
    x, tokens = make(n, V, dtype, seed=V + n)
    check(x, tokens)
    check(x, tokens, top=min(V, 20), tau=0.7)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (3, 5), (8, 8), (7, 2)])
def test_rows_at_any_address(dtype, pad, offset):
    x, tokens = make(5, 10_001, dtype, 3, pad, offset=offset)
    check(x, tokens, tau=2.0)
    check(x, tokens, top=37, tau=2.0)


def test_one_row_again_and_again():
    x, tokens = make(1, 5003, BF16, 1)
    check(x.expand(6, 5003), tokens.repeat(6))


@pytest.mark.parametrize("top", [0, 5])
def test_tokens_outside_the_vocabulary_are_padding(top):
    x, tokens = make(6, 999, F32, 4)
    tokens[:5] = torch.tensor([-1, 999, -100, 2**31 - 1, -(2**31)])
    got = check(x, tokens, top=top)
    assert got.logprobs[:5].tolist() == [0.0] * 5


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap", [2.0, 8.0, 20.0, 60.0])
@pytest.mark.parametrize("most", [1, 3])
def test_rows_that_are_nearly_sure(dtype, gap, most):
    """Entropies and log probabilities down to 10^-20 keep their places."""
    V = 30_011
    x, tokens = make(8, V, dtype, 5, spread=1.0)
    top = x.double().max(1, keepdim=True).values
    for r in range(8):
        at = torch.randperm(V, generator=torch.Generator().manual_seed(r))[:most].cuda()
        x[r, at] = (top[r] + gap + math.log(V)).to(dtype)
        if r % 2:
            tokens[r] = at[0]
    check(x, tokens)
    check(x, tokens, top=4)


def special(dtype):
    V = 20_000
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    g = torch.Generator().manual_seed(5)
    x = torch.randn(14, V, generator=g).to(dtype)
    x[0] = 1.5
    x[1] = -INF
    x[2, 5:] = -INF
    x[3] = low
    x[4, 100:] = low
    x[5, ::2] = -INF
    x[6, 777] = NAN
    x[7, [3, 19_999]] = INF
    x[8, 19_999] = 50.0
    x[9] = high
    x[10] = torch.arange(V).to(dtype)
    x[11, :4000] = 9.0
    x[12, :] = -INF
    x[12, 7] = NAN
    x[13, 5:] = low
    tokens = torch.tensor([4, 9, 6, 19_999, 50, 0, 3, 3, 19_999, 1, 19_999, 4000, 8, 2], dtype=torch.int32)
    return x.cuda(), tokens.cuda()


@pytest.mark.parametrize("repeat", [1, 60])
@pytest.mark.parametrize("top", [0, 7])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_special_rows(dtype, top, repeat):
    x, tokens = special(dtype)
    x, tokens = x.repeat(repeat, 1), tokens.repeat(repeat)
    got = rows.token_logprobs(x, tokens, top=top)
    kind = torch.arange(len(tokens), device="cuda") % 14
    masked, wild = kind == 1, (kind == 6) | (kind == 7) | (kind == 12)
    plain = ~masked & ~wild
    log_q, lp, lp_tol, entropy, entropy_tol = reference(x[plain], tokens[plain], 1.0)
    close(got.logprobs[plain], lp, lp_tol)
    close(got.entropy[plain], entropy, entropy_tol)
    assert bool((got.logprobs[masked] == -INF).all()) and bool((got.entropy[masked] == 0).all())
    assert bool(torch.isnan(got.logprobs[wild]).all()) and bool(torch.isnan(got.entropy[wild]).all())
    if top:
        ids, values, _ = rows.top_logits(x, top)
        assert torch.equal(got.ids, ids)
        assert bool((got.alternatives[ids < 0] == -INF).all())
        assert bool(torch.isnan(got.alternatives[wild & (kind != 12)]).all())
    w = torch.ones(len(tokens), device="cuda")
    grad = rows.token_logprobs_grad(x, tokens, got.stats, w, w)
    assert not bool(grad[masked].any()) and bool(torch.isnan(grad[wild].float()).all(1).all()) and bool(torch.isfinite(grad[plain].float()).all())
    w[wild] = 0.0
    assert not bool(rows.token_logprobs_grad(x, tokens, got.stats, w, w)[wild].any())         # a row of weights 0


def test_rows_far_from_zero():
    """Logits around 10^7 and temperatures that leave no room for a whole reference."""
    x, tokens = make(6, 4000, F32, 8)
    check(x * 4 + 1e7, tokens)
    check(x * 4 - 1e7, tokens, top=5)
    for tau in (1e-6, 1e-3, 1e3, 1e6):
        check(x, tokens, tau=tau)
        check(x, tokens, top=3, tau=tau)


# --- gradient ----------------------------------------------------------------------------------------------------------------

def gradient(x, tokens, w, h, tau):
    """The formula in 64 bits, with its bound (module docstring; statistics are rounded to single precision on the way)."""
    log_q, lp, _, entropy, _ = reference(x, tokens, tau)
    x, q = x.double(), torch.exp(log_q)
    V = x.shape[1]
    known = (tokens >= 0) & (tokens < V)
    w, h = torch.where(known, w.double(), 0.0)[:, None], h.double()[:, None]
    m = x.max(1, keepdim=True).values
    d = torch.nan_to_num((m - x) / tau, nan=0.0, posinf=0.0)
    one = torch.zeros_like(x).scatter_(1, torch.where(known, tokens, 0).long()[:, None], known.double()[:, None])
    # 1 - q of the token from its logarithm
    other = torch.where(one > 0, -torch.expm1(lp)[:, None], -q)
    mean = (q * d).sum(1, keepdim=True)
    log_z = (entropy[:, None] - mean).clamp(min=0)
    g = (w * other + h * torch.where(q > 0, -q * (mean - d), 0.0)) / tau
    delta = 2.0**-22 * (2 + 1.4427 * d) + 2.0**-23 * (1 + log_z)
    tol = (w.abs() * (q * delta + 2.0**-22 * other.abs()) + h.abs() * q * (mean + d) * (delta + 2.0**-21)) / tau
    return g, tol


def check_grad(x, tokens, tau=1.0, w=None, h=None, grad=None):
    n = x.shape[0]
    g = torch.Generator().manual_seed(n)
    w = torch.randn(n, generator=g).cuda() if w is None else w
    h = (0.1 * torch.randn(n, generator=g)).cuda() if h is None else h
    stats = rows.token_logprobs(x, tokens, temperature=tau).stats
    want, tol = gradient(x, tokens, w, h, tau)
    got = rows.token_logprobs_grad(x, tokens, stats, w, h, temperature=tau, grad=grad)
    dtype = x.dtype
    close(got, want, tol * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * want.abs() + SMALLEST[dtype])
    return got


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,V", SIZES[:-3] + [(70, 40_000)])
def test_gradient(n, V, dtype):
    x, tokens = make(n, V, dtype, seed=V + 2 * n)
    check_grad(x, tokens, tau=0.8)


def test_gradient_of_weights_left_out_and_zero():
    x, tokens = make(4, 3000, F32, 1)
    zero, one = torch.zeros(4, device="cuda"), torch.ones(4, device="cuda")
    stats = rows.token_logprobs(x, tokens).stats
    for w, h in ((one, None), (None, one), (None, None)):
        want, tol = gradient(x, tokens, zero if w is None else w, zero if h is None else h, 1.0)
        close(rows.token_logprobs_grad(x, tokens, stats, w, h), want, tol + HALF_STEP[F32] * want.abs() + SMALLEST[F32])
    tokens[0] = -1                         # padding has no weight
    check_grad(x, tokens)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad,offset,grad_pad", [(0, 0, 3), (1, 0, 1), (5, 3, 0), (8, 8, 8), (2, 1, 7)])
def test_gradient_of_rows_at_any_address(dtype, pad, offset, grad_pad):
    x, tokens = make(5, 10_001, dtype, 3, pad, offset=offset)
    wide = torch.full((5, 10_001 + grad_pad), 7.0, dtype=dtype, device="cuda")
    check_grad(x, tokens, grad=wide[:, :10_001])
    assert bool((wide[:, 10_001:] == 7.0).all())
    before = x.clone()
    want = rows.token_logprobs_grad(before, tokens, rows.token_logprobs(x, tokens).stats, torch.ones(5, device="cuda"))
    got = rows.token_logprobs_grad(x, tokens, rows.token_logprobs(x, tokens).stats, torch.ones(5, device="cuda"), grad=x)      # in the logits' place
    assert got is x and torch.equal(x, want)


@pytest.mark.parametrize("gap", [3.0, 12.0, 40.0])
def test_gradient_of_rows_that_are_nearly_sure(gap):
    V = 20_011
    x, tokens = make(6, V, F32, 5, spread=1.0)
    for r in range(6):
        x[r, 11 * r] = x[r].max() + gap + math.log(V)
        if r % 2:
            tokens[r] = 11 * r
    check_grad(x, tokens)


def test_gradient_against_differences():
    """Central differences with a step of 1/16: off by (1/16)^2 / 6 of the third derivative (below 1/4 for both), and by 2^-21 of the values (up
    to 8) over the step."""
    x, tokens = make(1, 40, F32, 2, spread=1.0)
    step = 1 / 16
    eye = step * torch.eye(40, device="cuda")
    up, down = rows.token_logprobs(x + eye, tokens.repeat(40)), rows.token_logprobs(x - eye, tokens.repeat(40))
    stats, one = rows.token_logprobs(x, tokens).stats, torch.ones(1, device="cuda")
    for i, args in enumerate(((one, None), (None, one))):
        got = rows.token_logprobs_grad(x, tokens, stats, *args)[0]
        want = (up[i] - down[i]) / (2 * step)
        assert float((got - want).abs().max()) <= step**2 / 6 / 4 + 2.0**-21 * 8 / step


def test_autograd():
    x, tokens = make(9, 3000, BF16, 6)
    leaf = x.detach().clone().requires_grad_()
    w, h = torch.randn(9, device="cuda"), torch.randn(9, device="cuda")
    got = rows.token_logprobs(leaf, tokens, top=3, temperature=1.3)
    assert got.logprobs.requires_grad and got.entropy.requires_grad
    assert not any(t.requires_grad for t in (got.stats, got.ids, got.alternatives))
    both, = torch.autograd.grad([got.logprobs, got.entropy], [leaf], [w, h], retain_graph=True)
    assert torch.equal(both, rows.token_logprobs_grad(x, tokens, got.stats, w, h, temperature=1.3))
    one, = torch.autograd.grad([got.logprobs], [leaf], [w], retain_graph=True)
    assert torch.equal(one, rows.token_logprobs_grad(x, tokens, got.stats, w, None, temperature=1.3))
    # broadcast inputs, and weights that autograd hands over with stride 0
    one = x[:1].detach().clone().requires_grad_()
    rows.token_logprobs(one.expand(4, 3000), tokens[:4]).logprobs.sum().backward()
    each = rows.token_logprobs_grad(x[:1].expand(4, 3000), tokens[:4], rows.token_logprobs(x[:1].expand(4, 3000), tokens[:4]).stats, torch.ones(4, device="cuda"))
    bound = 4 * 4 * HALF_STEP[BF16] * each.float().abs().sum(0) + 2.0**-130       # sums of four bf16 numbers, rounded along the way
    assert bool(((one.grad[0].float() - each.float().sum(0)).abs() <= bound).all())
    # a gradient written over saved logits is noticed
    kept = rows.token_logprobs(leaf, tokens)
    rows.token_logprobs_grad(leaf, tokens, kept.stats, w, grad=leaf.detach())
    with pytest.raises(RuntimeError, match="modified"):
        kept.logprobs.sum().backward()


# --- streams and graphs, and the operators together --------------------------------------------------------------------------

def test_a_replayed_graph_and_another_stream():
    x, tokens = make(33, 7001, BF16, 12)
    w = torch.randn(33, device="cuda")

    def call():
        got = rows.token_logprobs(x, tokens, top=9)
        return (*got, rows.token_logprobs_grad(x, tokens, got.stats, w, w))

    want = call()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    x.copy_(make(33, 7001, BF16, 13)[0])
    want = call()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(out, want))


@pytest.mark.parametrize("captured", [False, True])
def test_the_targets_pass_over_drafts(captured):
    """What a server does with drafts, as one run: their keys into the cache, attention of the chains and of trees, verification against the
    target's probabilities, and what is reported of the tokens that stand."""
    g = torch.Generator().manual_seed(3)
    n, heads, kv_heads, dim, page, V = 5, 8, 2, 64, 16, 3001
    drafts_of = [3, 0, 5, 1, 4]
    contexts = [40, 700, 15, 0, 130]
    new = [d + 1 for d in drafts_of]                        # the last token of the text, then its drafts
    tokens, drafts = sum(new), sum(drafts_of)
    offsets = torch.tensor([sum(new[:i]) for i in range(n + 1)]).cuda()
    draft_offsets = torch.tensor([sum(drafts_of[:i]) for i in range(n + 1)]).cuda()
    starts = torch.tensor(contexts, dtype=torch.int32).cuda()
    need = [-(-(c + m) // page) for c, m in zip(contexts, new)]
    order = torch.randperm(sum(need), generator=g).to(torch.int32)
    table = torch.full((n, max(need)), -1, dtype=torch.int32)
    for i, k in enumerate(need):
        table[i, :k], order = order[:k], order[k:]
    table = table.cuda()
    k_cache, v_cache = (torch.randn(sum(need), page, kv_heads, dim, generator=g).to(BF16).cuda() for _ in range(2))
    q, k, v = (torch.randn(tokens, h, dim, generator=g).to(BF16).cuda() for h in (heads, kv_heads, kv_heads))
    parents = torch.cat([torch.arange(m) - 1 for m in new]).to(torch.int32).cuda()
    inv_freq = (1e4 ** (-torch.arange(0, dim, 2).double() / dim)).float().cuda()
    head = (torch.randn(heads * dim, V, generator=g) / 16).cuda()
    words = torch.randint(0, V, (drafts,), generator=g).to(torch.int32).cuda()
    accept_u, draw_u = torch.rand(drafts, generator=g).cuda() * 2e-3, torch.rand(n, generator=g).cuda()

    def call():
        mask, positions = cache.tree_mask(parents, offsets, starts, max(new))
        turned = cache.append_cache(k, v, k_cache, v_cache, table, starts, offsets, positions=positions, inv_freq=inv_freq, q=q)
        out = cache.tree_attention(turned, k_cache, v_cache, table, starts, offsets, mask=mask)
        logits = out.float().flatten(1) @ head
        picked, accepted = rows.verify_drafts(draft_offsets, words, torch.softmax(logits, 1), None, accept_u, draw_u)
        return mask, positions, turned, out, logits, picked, accepted, rows.token_logprobs(logits, picked, top=5)

    first = call()
    chain = cache.tree_attention(first[2], k_cache, v_cache, table, starts, offsets)         # a chain is what no mask says
    assert torch.equal(first[3], chain)
    mask, positions, turned, out, logits, picked, accepted, got = first
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            later = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(later[:7], first[:7])) and all(torch.equal(a, c) for a, c in zip(later[7], got))
    place = torch.cat([torch.arange(m) for m in new]).cuda()
    seq = torch.repeat_interleave(torch.arange(n), torch.tensor(new)).cuda()
    assert torch.equal(positions, (starts[seq] + place).to(torch.int32)) and torch.equal(mask[:, 0], (2 << place) - 1)
    want = torch.zeros(tokens, heads, dim, dtype=torch.float64, device="cuda")
    for i in range(n):
        total = contexts[i] + new[i]
        s = torch.arange(total, device="cuda")
        keys, values = (c[table[i].long()[s // page], s % page].double().repeat_interleave(heads // kv_heads, 1) for c in (k_cache, v_cache))
        rows_ = slice(int(offsets[i]), int(offsets[i + 1]))
        score = torch.einsum("nhd,khd->hnk", turned[rows_].double(), keys) / dim**0.5
        score = score.masked_fill(s > contexts[i] + torch.arange(new[i], device="cuda")[:, None], -INF)
        want[rows_] = torch.einsum("hnk,khd->nhd", torch.softmax(score, -1), values)
    # (probabilities and outputs are rounded to bf16, each by 2^-8 at most of what is at most the largest value)
    assert float((out.double() - want).abs().max()) <= 3 * 2.0**-8 * float(v_cache.double().abs().max())
    log_q = torch.log_softmax(logits.double(), 1)
    there = picked >= 0
    assert bool((accepted >= 0).all()) and int(there.sum()) == int(accepted.sum()) + n
    close(got.logprobs[there], torch.gather(log_q, 1, picked.long().clamp(min=0)[:, None])[there, 0], torch.full((int(there.sum()),), 2.0**-18))
    assert bool((got.logprobs[~there] == 0).all())
