"""The target's pass over drafted tokens and what is reported of them, as measurable cases.

Kinds of work (field "op"):

mask     trees of drafted tokens, given by every node's parent: who sees whom, as bits, and the nodes' positions.
append   new tokens' keys and values into a paged cache, with the position rotation of keys (and queries) on the way.
attend   attention of new tokens, a tree of them or one per sequence, over the paged cache.
logp     log probabilities of given tokens with the rows' entropies, with the largest alternatives ("top") or, for a training step, with
         the gradient of a weighted sum of both ("grad").

Vocabularies are those of synth.CONFIGS and of perf/operators.py; heads and pages are generic.  Contexts and trees are ragged: every length
from about a quarter of the longest on.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZES = {"float32": 4, "float16": 2, "bfloat16": 2}


def _named(name, c):
    return dict(c, name=name) if name else c


def _mask(name, seqs, nodes, deep):
    return _named(name, dict(op="mask", seqs=seqs, nodes=nodes, deep=deep))


def _append(name, seqs, new, context, heads, kv_heads, dim, rot, page, dtype, interleaved=False, queries=True):
    return _named(name, dict(op="append", seqs=seqs, new=new, context=context, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, page=page,
                             dtype=dtype, interleaved=interleaved, queries=queries))


def _attend(name, seqs, new, context, heads, kv_heads, dim, page, dtype, by_head=False):
    return _named(name, dict(op="attend", seqs=seqs, new=new, context=context, heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype,
                             by_head=by_head))


def _logp(name, rows, V, dtype, top=0, grad=False, pad=0, masked=False, tau=1.0):
    return _named(name, dict(op="logp", rows=rows, V=V, dtype=dtype, top=top, grad=grad, pad=pad, masked=masked, tau=tau))


def listed():
    return [
        # the trees of a serving batch
        _mask("mask_batch", 64, 48, False),
        # as many as one call may have in earnest, the largest trees, some of them one long chain
        _mask("mask_large", 2048, 255, True),
        # one decoding step of a batch: one token each, all latency
        _append("append_step", 32, 1, 2048, 32, 8, 128, 128, 16, "bfloat16"),
        # prompts in one piece
        _append("append_prompt", 4, 8192, 0, 32, 8, 128, 128, 64, "bfloat16"),
        # odd sizes: part of each head rotated, neighbours as pairs, drafts behind contexts
        _append("append_odd", 129, 37, 1021, 15, 5, 80, 32, 24, "float16", interleaved=True),
        # one sequence, a small tree over a long context
        _attend("attend_one", 1, 8, 32_768, 32, 8, 128, 16, "bfloat16"),
        # a decoding step: one token each
        _attend("attend_step", 64, 1, 8192, 32, 8, 128, 16, "bfloat16"),
        # trees of 64 nodes in a serving batch
        _attend("attend_tree", 16, 64, 8192, 32, 8, 128, 64, "bfloat16"),
        # odd sizes: a group of three, heads of 80, pages of 24, the cache kept head by head
        _attend("attend_odd", 33, 13, 2050, 15, 5, 80, 24, "float16", by_head=True),
        # what a served step reports
        _logp("logp_step", 8, 10_000, "float32", top=5),
        # a batch's sampled tokens with their alternatives, an odd vocabulary with masked words, rows at odd addresses
        _logp("logp_alternatives", 777, 100_003, "float16", top=20, pad=2, masked=True, tau=0.8),
        # a policy-gradient step: log probabilities and entropies with their gradient
        _logp("logp_train", 2048, 141_000, "bfloat16", grad=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["mask", "append", "attend", "attend", "logp"])
    if op == "mask":
        nodes = _log_int(rng, 2, 256)
        return _mask(None, _log_int(rng, 1, min(4096, 520_000 // nodes)), nodes, rng.random() < 0.3)
    if op == "logp":
        dtype = rng.choice(list(DTYPES))
        V = _log_int(rng, 500, 1_000_000)
        rows = _log_int(rng, 1, max(1, min(8192, 280_000_000 // V)))
        grad = rng.random() < 0.5
        top = 0 if grad or rng.random() < 0.4 else _log_int(rng, 1, min(512, V))
        return _logp(None, rows, V, dtype, top, grad, rng.choice([0, 0, 1, 2, 8, 13]), rng.random() < 0.4, rng.choice([0.7, 1.0, 1.0, 1.5]))
    dtype = rng.choice(["float16", "bfloat16"])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 16])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8])
    dim = rng.choice([64, 64, 80, 96, 128, 128, 256])
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    if op == "append":
        seqs = _log_int(rng, 1, 256)
        new = _log_int(rng, 1, max(1, min(8192, 80_000_000 // (seqs * heads * dim))))
        rot = rng.choice([dim, dim, dim // 2, 0])
        context = rng.choice([0, _log_int(rng, 1, max(1, min(32_768, 100_000_000 // (seqs * kv_heads * dim))))])
        return _append(None, seqs, new, context, heads, kv_heads, dim, rot, page, dtype, rng.random() < 0.4, rng.random() < 0.7)
    seqs = _log_int(rng, 1, 128)
    context = _log_int(rng, 1, max(1, min(65_536, 100_000_000 // (seqs * kv_heads * dim))))
    new = min(rng.choice([1, _log_int(rng, 2, 64)]), max(1, 25_000_000_000 // (seqs * heads * dim * (context + 64))))
    return _attend(None, seqs, new, context, heads, kv_heads, dim, page, dtype, rng.random() < 0.4)


# --- inputs ------------------------------------------------------------------------------------------------------------------

def _padded(x, pad):
    """x with rows that lie `pad` values further apart than they are long."""
    if not pad:
        return x.contiguous()
    wide = x.new_zeros(x.shape[0], x.shape[1] + pad)
    wide[:, : x.shape[1]] = x
    return wide[:, : x.shape[1]]


def _ragged(gen, seqs, most, least):
    """Lengths from `least` to `most`, about equally often, the longest among them, in any order."""
    i = torch.arange(seqs, device="cuda")
    return (most - i * (most - least) // max(1, seqs - 1))[torch.randperm(seqs, generator=gen, device="cuda")]


def _offsets(lengths):
    out = torch.zeros(lengths.numel() + 1, dtype=torch.int64, device="cuda")
    out[1:] = torch.cumsum(lengths, 0)
    return out


def _places(offsets):
    """Sequence of every new token, and its place there."""
    lengths = offsets[1:] - offsets[:-1]
    seq = torch.repeat_interleave(torch.arange(lengths.numel(), device="cuda"), lengths)
    return seq, torch.arange(seq.numel(), device="cuda") - offsets[seq]


def _parents(gen, offsets, deep):
    """Trees as drafters make them: most nodes hang on one of the last few, some on the root; every fourth one chain (deep)."""
    seq, place = _places(offsets)
    n = seq.numel()
    u = torch.rand(n, generator=gen, device="cuda")
    back = 1 + (8 * u * u).long()
    parent = place - back
    if deep:
        parent = torch.where(seq % 4 == 0, place - 1, parent)
    return parent.clamp(min=-1).to(torch.int32)


def _pages(gen, case, starts, new):
    """A cache's pages in no order, as many for every sequence as it needs, -1 behind them: (pages in all, table)."""
    page = case["page"]
    need = (starts + new + page - 1) // page
    width = max(1, int(need.max()))
    there = torch.arange(width, device="cuda") < need[:, None]
    # a few more than are needed: a number that the lengths' order does not change
    count = int(((starts + page - 1) // page + (new + page - 1) // page).sum())
    table = torch.full(there.shape, -1, dtype=torch.int32, device="cuda")
    table[there] = torch.randperm(count, generator=gen, device="cuda")[: int(need.sum())].to(torch.int32)
    return count, table


def _random(gen, shape, dtype, by=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype).mul_(by)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dev = "cuda"
    if case["op"] == "mask":
        offsets = _offsets(_ragged(gen, case["seqs"], case["nodes"], (case["nodes"] + 3) // 4))
        starts = torch.randint(0, 100_000, (case["seqs"],), generator=gen, device=dev).to(torch.int32)
        return dict(case=case, offsets=offsets, starts=starts, parents=_parents(gen, offsets, case["deep"]))
    if case["op"] == "logp":
        return _prepare_logp(case, gen)
    dt, dim, kv_heads, heads = DTYPES[case["dtype"]], case["dim"], case["kv_heads"], case["heads"]
    context = case["context"]
    starts = _ragged(gen, case["seqs"], context, (context + 3) // 4)
    new = _ragged(gen, case["seqs"], case["new"], (case["new"] + 3) // 4)
    offsets = _offsets(new)
    tokens = int(offsets[-1])
    pages, table = _pages(gen, case, starts, new)
    state = dict(case=case, offsets=offsets, table=table, starts=starts.to(torch.int32))
    if case["op"] == "append":
        # the three parts of one projection's rows
        rows = _random(gen, (tokens, (heads + 2 * kv_heads) * dim), dt)
        q, k, v = rows.split([heads * dim, kv_heads * dim, kv_heads * dim], 1)
        state.update(q=q.view(tokens, heads, dim) if case["queries"] else None, k=k.view(tokens, kv_heads, dim), v=v.view(tokens, kv_heads, dim))
        for name in ("k_cache", "v_cache"):
            state[name] = _random(gen, (pages, case["page"], kv_heads, dim), dt)
        seq, place = _places(offsets)
        state["positions"] = (starts[seq] + place).to(torch.int32)
        state["inv_freq"] = None
        if case["rot"]:
            state["inv_freq"] = (1e6 ** (-torch.arange(0, case["rot"], 2, device=dev).double() / case["rot"])).float()
        return state
    shape = (pages, kv_heads, case["page"], dim) if case["by_head"] else (pages, case["page"], kv_heads, dim)
    for name in ("k_cache", "v_cache"):
        cache = _random(gen, shape, dt)
        state[name] = cache.transpose(1, 2) if case["by_head"] else cache
    state["q"] = _random(gen, (tokens, heads, dim), dt, 1.5)
    # the mask of the drafted trees, made once for all layers
    state["mask"] = _plain_mask(offsets, state["starts"], _parents(gen, offsets, False), case["new"])["mask"] if case["new"] > 1 else None
    return state


def _prepare_logp(case, gen):
    dt, V, n, dev = DTYPES[case["dtype"]], case["V"], case["rows"], "cuda"
    # logits as a model of text gives them: a bias that falls with the word's rank (words in no order), a normal part per place, and
    # a few words that this place makes likely
    rank = torch.randperm(V, generator=gen, device=dev).float()
    x = torch.randn(n, V, generator=gen, device=dev)
    x.mul_(2.0).sub_(torch.log1p(rank))
    few = min(8, V)
    at = torch.randint(V, (n, few), generator=gen, device=dev)
    x.scatter_add_(1, at, 6 + 8 * torch.rand(n, few, generator=gen, device=dev))
    if case["masked"]:
        x.masked_fill_(torch.rand(V, generator=gen, device=dev) < 1 / 16, -math.inf)
    logits = x.to(dt, copy=True)
    # sampled: the largest logit plus Gumbel noise
    u = torch.rand(n, V, generator=gen, device=dev).clamp_(min=1e-30)
    tokens = x.div_(case["tau"]).sub_(u.log_().neg_().clamp_(min=1e-30).log_()).argmax(1).to(torch.int32)
    state = dict(case=case, logits=_padded(logits, case["pad"]), tokens=tokens)
    if case["grad"]:
        scale = (65536.0 if dt == torch.float16 else 1.0) / n
        state["logits"].requires_grad_()
        state["d_logprobs"] = torch.randn(n, generator=gen, device=dev) * scale      # advantages
        state["d_entropy"] = torch.full((n,), 0.01 * scale, device=dev)
    return state


# --- the framework's calls ---------------------------------------------------------------------------------------------------

def _own(s):
    from paper_1412_1576_b200 import cache, rows
    case = s["case"]
    if case["op"] == "mask":
        mask, positions = cache.tree_mask(s["parents"], s["offsets"], s["starts"], case["nodes"])
        return dict(mask=mask, positions=positions)
    if case["op"] == "append":
        q = cache.append_cache(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["offsets"], positions=s["positions"],
                               inv_freq=s["inv_freq"], interleaved=case["interleaved"], q=s["q"])
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"], q=q) if q is not None else dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    if case["op"] == "attend":
        return dict(out=cache.tree_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["starts"], s["offsets"], mask=s["mask"]))
    got = rows.token_logprobs(s["logits"], s["tokens"], top=case["top"], temperature=case["tau"])
    if case["grad"]:
        grad, = torch.autograd.grad([got.logprobs, got.entropy], [s["logits"]], [s["d_logprobs"], s["d_entropy"]])
        return dict(logprobs=got.logprobs.detach(), entropy=got.entropy.detach(), grad=grad)
    if case["top"]:
        return dict(logprobs=got.logprobs, entropy=got.entropy, ids=got.ids, alternatives=got.alternatives)
    return dict(logprobs=got.logprobs, entropy=got.entropy)


# --- the plain forms ---------------------------------------------------------------------------------------------------------

def _plain_mask(offsets, starts, parents, nodes):
    seq, place = _places(offsets)
    n, words = seq.numel(), (nodes + 63) // 64
    dev = offsets.device
    # node by node along the parents: the steps of all trees at a time, until every node has reached its root
    at = place.clone()
    mask = torch.zeros(n, words, dtype=torch.int64, device=dev)
    depth = torch.full((n,), -1, dtype=torch.int64, device=dev)
    word = torch.arange(words, device=dev)
    while bool((at >= 0).any()):
        here = at >= 0
        bit = torch.where(here, torch.ones_like(at) << (at % 64), 0)
        mask |= torch.where(word == (at // 64)[:, None], bit[:, None], 0)
        depth += here
        at = torch.where(here, parents[(offsets[seq] + at).clamp(min=0)].long(), -1)
    return dict(mask=mask, positions=(starts[seq] + depth).to(torch.int32))


def _rotated(x, positions, inv_freq, interleaved):
    """x: [tokens, heads, dim]; its first 2 * inv_freq.numel() values of a head are rotated."""
    x = x.float()
    if inv_freq is None:
        return x
    half = inv_freq.numel()
    angle = positions.double()[:, None] * inv_freq.double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = (x[..., 0 : 2 * half : 2], x[..., 1 : 2 * half : 2]) if interleaved else (x[..., :half], x[..., half : 2 * half])
    pair = (a * cos - b * sin, a * sin + b * cos)
    turned = torch.stack(pair, -1).flatten(-2) if interleaved else torch.cat(pair, -1)
    return torch.cat([turned, x[..., 2 * half :]], -1)


def _plain_append(case, s):
    seq, place = _places(s["offsets"])
    slot = s["starts"][seq].long() + place
    page = s["table"][seq, slot // case["page"]].long()
    dt = s["k_cache"].dtype
    s["k_cache"][page, slot % case["page"]] = _rotated(s["k"], s["positions"], s["inv_freq"], case["interleaved"]).to(dt)
    s["v_cache"][page, slot % case["page"]] = s["v"]
    out = dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    if s["q"] is not None:
        out["q"] = _rotated(s["q"], s["positions"], s["inv_freq"], case["interleaved"]).to(dt)
    return out


def _plain_attend(case, s):
    offsets, starts, dev = s["offsets"], s["starts"].long(), s["q"].device
    seqs, new, kv_heads, dim, page = case["seqs"], case["new"], case["kv_heads"], case["dim"], case["page"]
    group = case["heads"] // kv_heads
    seq, place = _places(offsets)
    total = starts + offsets[1:] - offsets[:-1]
    width = s["table"].shape[1] * page
    key = torch.arange(width, device=dev)
    slots = s["table"].long().clamp(min=0)[:, key // page] * page + key % page
    def of(cache):
        return cache.reshape(-1, kv_heads, dim)[slots].float().transpose(1, 2)
    q = torch.zeros(seqs, new, kv_heads, group, dim, device=dev)
    q[seq, place] = s["q"].float().view(-1, kv_heads, group, dim)
    q = q.permute(0, 2, 1, 3, 4).reshape(seqs, kv_heads, new * group, dim)
    # the context, and of the new tokens those that the mask names (without one: those up to its own place)
    seen = torch.zeros(seqs, new, width, dtype=torch.bool, device=dev)
    j = key - starts[seq][:, None]
    if s["mask"] is None:
        bits = j <= place[:, None]
    else:
        bits = (torch.gather(s["mask"], 1, (j // 64).clamp(0, s["mask"].shape[1] - 1)) >> (j % 64)) & 1 == 1
    seen[seq, place] = (key < total[seq][:, None]) & ((j < 0) | bits)
    scores = torch.matmul(q, of(s["k_cache"]).transpose(2, 3)) / math.sqrt(dim)
    scores = scores.view(seqs, kv_heads, new, group, width).masked_fill_(~seen[:, None, :, None], -math.inf)
    scores -= scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = scores.exp_()
    norm = p.sum(-1, keepdim=True)
    v = of(s["v_cache"]).masked_fill_((key >= total[:, None])[:, None, :, None], 0.0)
    out = torch.matmul(p.view(seqs, kv_heads, new * group, width), v).view(seqs, kv_heads, new, group, dim)
    out = torch.where(norm > 0, out / norm, 0.0).permute(0, 2, 1, 3, 4)[seq, place]
    return dict(out=out.reshape(-1, case["heads"], dim).to(s["q"].dtype))


def _ordered(x):
    """Whole numbers in the order of the values (NaN above all, both zeros alike)."""
    b = (x + 0.0).view(torch.int32)
    return torch.where(torch.isnan(x), 0x7FFFFFFF, b ^ ((b >> 31) & 0x7FFFFFFF))


def _plain_logp(case, s):
    tau = case["tau"]
    logits = s["logits"].detach()
    x = logits.float()
    at = s["tokens"].long()[:, None]
    m = x.max(1, keepdim=True).values
    y = (x - m) / tau
    e = torch.exp(y)
    # the sum without the largest, which is 1: what is left of a row that is nearly sure would be lost beside it
    rest = torch.where(y < 0, e, 0.0).double().sum(1)
    most = (y == 0).sum(1).double()
    log_z = torch.log1p(most - 1 + rest)
    z = most + rest
    spread = torch.where(e > 0, e * y, 0.0).double().sum(1) / z
    token = (torch.gather(x, 1, at) - m)[:, 0].double() / tau
    logprobs, entropy = token - log_z, log_z - spread
    out = dict(logprobs=logprobs.float(), entropy=entropy.float())
    if case["grad"]:
        w, h = s["d_logprobs"].double(), s["d_entropy"].double()
        by_q = (-w - h * (entropy - log_z)) / (z * tau)
        g = torch.where(e > 0, e * (by_q.float()[:, None] - (h / (z * tau)).float()[:, None] * y), 0.0)
        # (1 - q of a likely token from its logarithm)
        own_q = torch.exp(logprobs)
        there = (-torch.expm1(logprobs) * w - own_q * h * (logprobs + entropy)) / tau
        g.scatter_(1, at, there.float()[:, None])
        out["grad"] = g.to(logits.dtype)
    if case["top"]:
        V, dev = case["V"], x.device
        key = _ordered(x).long() * 2**32 + (2**32 - 1 - torch.arange(V, device=dev))
        ids = torch.topk(key, case["top"], dim=1).indices
        del key
        values = torch.gather(x, 1, ids)
        out["ids"] = ids.masked_fill(values == -math.inf, -1).to(torch.int32)
        out["alternatives"] = ((values - m).double() / tau - log_z[:, None]).float()
    return out


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["op"] == "mask":
        return _plain_mask(state["offsets"], state["starts"], state["parents"], case["nodes"])
    if case["op"] == "append":
        return _plain_append(case, state)
    return _plain_attend(case, state) if case["op"] == "attend" else _plain_logp(case, state)


def _mean(most):
    """Average of the lengths that _ragged gives, about."""
    return (most + (most + 3) // 4) / 2


def work(case):
    if case["op"] == "mask":
        nodes = case["seqs"] * _mean(case["nodes"])
        return dict(bytes=nodes * (8 + 8 * ((case["nodes"] + 63) // 64)) + case["seqs"] * 12, flops=nodes * 8)
    size = SIZES[case["dtype"]]
    if case["op"] == "logp":
        rows, V = case["rows"], case["V"]
        return dict(bytes=rows * (V * size * (2 if case["grad"] else 1) + 8 * case["top"] + 12 + (8 if case["grad"] else 0)),
                    flops=rows * V * (12 if case["grad"] else 6))
    tokens = case["seqs"] * (_mean(case["new"]) if case["seqs"] > 1 else case["new"])
    context = case["seqs"] * (_mean(case["context"]) if case["seqs"] > 1 else case["context"])
    dim, heads, kv_heads = case["dim"], case["heads"], case["kv_heads"]
    if case["op"] == "append":
        moved = 2 * kv_heads + (heads if case["queries"] else 0)
        return dict(bytes=tokens * (2 * moved * dim * size + 8), flops=tokens * (moved - kv_heads) * case["rot"] * 3)
    # (longest contexts and trees lie in no order beside each other)
    pairs = tokens * context / case["seqs"] + tokens * _mean(case["new"]) / 2
    return dict(bytes=(2 * (context + tokens) * kv_heads + 2 * tokens * heads) * dim * size + case["seqs"] * case["context"] / case["page"] * 4,
                flops=4 * pairs * heads * dim)


# --- the operators' definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_mask(case, s):
    offsets, parents, starts = s["offsets"].tolist(), s["parents"].tolist(), s["starts"].tolist()
    words = (case["nodes"] + 63) // 64
    mask, positions = [], []
    for b in range(case["seqs"]):
        bits, depth = [], []
        for i in range(offsets[b + 1] - offsets[b]):
            parent = parents[offsets[b] + i]
            bits.append((bits[parent] if parent >= 0 else 0) | 1 << i)
            depth.append(depth[parent] + 1 if parent >= 0 else 0)
        mask += [[(x >> 64 * w & (1 << 64) - 1) - (x >> 64 * w + 63 & 1) * (1 << 64) for w in range(words)] for x in bits]
        positions += [starts[b] + d for d in depth]
    return dict(mask=torch.tensor(mask, dtype=torch.int64), positions=torch.tensor(positions, dtype=torch.int32))


def _exact_turn(x, position, inv_freq, interleaved):
    """Rotation of every pair as a product of complex numbers; x: [tokens, heads, dim] in 64 bits."""
    if inv_freq is None:
        return x
    n = inv_freq.numel()
    part = x[..., : 2 * n].reshape(*x.shape[:-1], n, 2) if interleaved else torch.stack([x[..., :n], x[..., n : 2 * n]], -1)
    turn = torch.exp(1j * (position.double()[:, None] * inv_freq.double()))[:, None]
    part = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
    out = x.clone()
    if interleaved:
        out[..., : 2 * n] = part.reshape(*x.shape[:-1], 2 * n)
    else:
        out[..., :n], out[..., n : 2 * n] = part[..., 0], part[..., 1]
    return out


def _exact_append(case, s):
    offsets, starts, table = s["offsets"].tolist(), s["starts"].tolist(), s["table"]
    k = _exact_turn(s["k"].double(), s["positions"], s["inv_freq"], case["interleaved"])
    caches = dict(k_cache=s["k_cache"].double(), v_cache=s["v_cache"].double())
    for b in range(case["seqs"]):
        lo, hi = offsets[b], offsets[b + 1]
        slot = torch.arange(starts[b], starts[b] + hi - lo, device=k.device)
        at = table[b].long()[slot // case["page"]] * case["page"] + slot % case["page"]
        caches["k_cache"].view(-1, case["kv_heads"], case["dim"])[at] = k[lo:hi]
        caches["v_cache"].view(-1, case["kv_heads"], case["dim"])[at] = s["v"][lo:hi].double()
    if s["q"] is not None:
        caches["q"] = _exact_turn(s["q"].double(), s["positions"], s["inv_freq"], case["interleaved"])
    return caches


def _exact_attend(case, s):
    offsets, starts = s["offsets"].tolist(), s["starts"].tolist()
    heads, kv_heads, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(offsets[-1], heads, dim, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        lo, hi, before = offsets[b], offsets[b + 1], starts[b]
        n = hi - lo
        pages = s["table"][b, : (before + n + page - 1) // page].long()
        see = torch.ones(n, before + n, dtype=torch.bool, device="cuda")
        place = torch.arange(n, device="cuda")
        if s["mask"] is None:
            see[:, before:] = place[:, None] >= place
        else:
            see[:, before:] = s["mask"][lo:hi][:, place // 64] >> place % 64 & 1 == 1
        for h in range(kv_heads):
            k = s["k_cache"][pages, :, h].reshape(-1, dim)[: before + n].double()
            v = s["v_cache"][pages, :, h].reshape(-1, dim)[: before + n].double()
            mine = slice(h * heads // kv_heads, (h + 1) * heads // kv_heads)
            score = torch.einsum("ngd,kd->gnk", s["q"][lo:hi, mine].double(), k) / dim**0.5
            out[lo:hi, mine] = torch.einsum("gnk,kd->ngd", torch.softmax(score.masked_fill(~see, -math.inf), -1), v)
    return dict(out=out)


def _exact_logp(case, s):
    tau, n, V = case["tau"], case["rows"], case["V"]
    out = dict(logprobs=torch.zeros(n, dtype=torch.float64, device="cuda"), entropy=torch.zeros(n, dtype=torch.float64, device="cuda"))
    if case["grad"]:
        out["grad"] = torch.zeros(n, V, dtype=torch.float64, device="cuda")
    if case["top"]:
        out["ids"] = torch.zeros(n, case["top"], dtype=torch.int32, device="cuda")
        out["alternatives"] = torch.zeros(n, case["top"], dtype=torch.float64, device="cuda")
    step = max(1, 100_000_000 // V)
    for lo in range(0, n, step):
        x = s["logits"].detach()[lo : lo + step].double()
        log_q = torch.log_softmax(x / tau, 1)
        q = torch.exp(log_q)
        terms = torch.where(q > 0, -q * log_q, 0.0)
        at = s["tokens"][lo : lo + step].long()[:, None]
        out["logprobs"][lo : lo + step] = torch.gather(log_q, 1, at)[:, 0]
        out["entropy"][lo : lo + step] = terms.sum(1)
        if case["grad"]:
            w, h = s["d_logprobs"][lo : lo + step, None].double(), s["d_entropy"][lo : lo + step, None].double()
            g = h * (terms - q * terms.sum(1, keepdim=True)) - w * q
            out["grad"][lo : lo + step] = g.scatter_add_(1, at, w) / tau
        if case["top"]:
            values, ids = torch.sort(x, dim=1, descending=True, stable=True)
            values, ids = values[:, : case["top"]], ids[:, : case["top"]]
            out["ids"][lo : lo + step] = ids.masked_fill(values == -math.inf, -1).to(torch.int32)
            out["alternatives"][lo : lo + step] = torch.gather(log_q, 1, ids)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "mask":
        return _exact_mask(case, s)
    if case["op"] == "append":
        return _exact_append(case, s)
    return _exact_attend(case, s) if case["op"] == "attend" else _exact_logp(case, s)
