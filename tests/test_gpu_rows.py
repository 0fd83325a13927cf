"""The operators on rows of logits and probabilities against plain forms in 64 bits.

Tolerances.  With tau the temperature, V words, c = log2(e) / tau and m a row's maximum the kernels work out 2^((x - m) c):
x - m and its product are rounded (2^-24 each, relative to a number of at most |(x - m) c|), so is c itself, and the exponential is
2^-22 off at most, or zero where it is less than 2^-126 (a row's maximum gives 1, so a share q loses no more than that).  A sum of positive terms whose longest chain of additions has `DEPTH` steps adds DEPTH 2^-24, relative.
"""
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_1412_1576_b200 import binding as b
from paper_1412_1576_b200 import rows

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF_STEP = {F32: 2.0**-24, F16: 2.0**-11, BF16: 2.0**-8}
SMALLEST = {F32: 2.0**-150, F16: 2.0**-25, BF16: 2.0**-134}      # half the distance of the numbers around zero
DEPTH = 160
NAN, INF = float("nan"), float("inf")


def make(n_rows, V, dtype, seed, pad=0, spread=3.0, offset=0):
    """Logits on the GPU: row stride V + pad, first element `offset` elements into its buffer."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n_rows, V, generator=g) * spread).to(dtype)
    flat = torch.full((offset + n_rows * (V + pad),), 77.0, dtype=dtype, device="cuda")
    view = flat[offset:].view(n_rows, V + pad)[:, :V]
    view.copy_(x)
    return view


def lse_error(x, tau):
    """Bound of the relative error of a row's sum of exponentials (x in 64 bits, on the CPU)."""
    far = torch.nan_to_num((x.max(1, keepdim=True).values - x) / tau, nan=0.0, posinf=0.0)
    q = torch.nan_to_num(torch.softmax(x / tau, 1), nan=0.0)
    return 2.0**-22 + 3 * 2.0**-24 * (q * far).sum(1) * 1.4427 + DEPTH * 2.0**-24


# --- top logits --------------------------------------------------------------------------------------------------------------

def top_reference(x, top, tau):
    """x: [rows, V] on the CPU."""
    d = x.double()
    V = x.shape[1]
    key = torch.where(torch.isnan(d), torch.full_like(d, INF), d)
    # two stable sorts: value descending, NaN before infinity
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    nan = torch.gather(torch.isnan(d), 1, order)
    order = torch.gather(order, 1, torch.sort(nan.to(torch.int8), dim=1, descending=True, stable=True).indices)
    ids = torch.full((x.shape[0], top), -1, dtype=torch.int32)
    values = torch.full((x.shape[0], top), -INF, dtype=x.dtype)
    k = min(top, V)
    at = order[:, :k]
    v = torch.gather(x, 1, at)
    ids[:, :k] = torch.where(v == -INF, -1, at).to(torch.int32)
    values[:, :k] = v
    return ids, values, torch.logsumexp(d / tau, 1)


def check_top(x, top, tau=1.0):
    ids, values, lse = rows.top_logits(x, top, temperature=tau)
    host = x.cpu()
    want_ids, want_values, want_lse = top_reference(host, top, tau)
    assert torch.equal(ids.cpu(), want_ids)
    assert torch.equal(torch.nan_to_num(values.cpu(), nan=1.0, posinf=2.0, neginf=3.0),
                       torch.nan_to_num(want_values, nan=1.0, posinf=2.0, neginf=3.0))
    got = lse.cpu().double()
    plain = torch.isfinite(want_lse)
    assert torch.equal(torch.isnan(got), torch.isnan(want_lse))
    assert torch.equal(got[~plain & ~torch.isnan(got)], want_lse[~plain & ~torch.isnan(got)])
    bound = lse_error(host.double(), tau) + 2.0**-23 + HALF_STEP[F32] * want_lse.abs()     # log of the sum: two units in the last place
    assert bool(((got - want_lse).abs() <= bound)[plain].all())


TOP_SIZES = [(1, 1, 1), (3, 1, 4), (5, 2, 2), (2, 7, 3), (4, 31, 31), (3, 32, 40), (2, 33, 1), (7, 255, 64), (3, 256, 256), (2, 1000, 512),
             (1, 4099, 20), (9, 10_000, 33), (300, 2_049, 5), (2, 50_021, 300), (3, 131_072, 64), (2, 141_000, 512), (1, 1_000_000, 128),
             (2, 1 << 20, 1)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n_rows,V,top", TOP_SIZES)
def test_top_logits(n_rows, V, top, dtype):
    check_top(make(n_rows, V, dtype, seed=V + top), top)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (3, 5), (8, 8), (7, 2)])
def test_top_logits_of_rows_at_any_address(dtype, pad, offset):
    check_top(make(5, 10_001, dtype, 3, pad, offset=offset), 37, tau=2.0)


@pytest.mark.parametrize("n_rows", [1, 2, 17, 147, 149, 600, 5000])
def test_top_logits_of_few_and_of_many_rows(n_rows):
    check_top(make(n_rows, 3_001, BF16, n_rows), 16, tau=0.7)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_many_rows_of_the_longest_vocabulary(dtype):
    """Enough rows for one CTA each: its share of the row is the largest there is."""
    V, n = 1 << 20, 1300
    one = make(1, V, dtype, 77)
    x = one.expand(n, V)
    ids, values, lse = rows.top_logits(x, 512)
    want = top_reference(one.cpu(), 512, 1.0)
    assert torch.equal(ids.cpu(), want[0].expand(n, 512)) and torch.equal(values.cpu(), want[1].expand(n, 512))
    assert bool((lse == lse[0]).all()) and abs(float(lse[0]) - float(want[2])) <= float(lse_error(one.cpu().double(), 1.0)) + 2.0**-20
    ids, values, teacher = lists_of(make(1, V, dtype, 78).cpu(), 512, 1.0, True, dtype)
    loss = rows.distill_loss(x, ids.expand(n, 512), values.expand(n, 512), teacher.repeat(n))
    want, tol, _, _ = distill_reference(one.cpu(), ids.cpu(), values.cpu(), teacher.cpu(), 1.0, torch.ones(1))
    assert bool((loss == loss[0]).all())
    same(loss[:1], want, tol, F32)


def special_rows(dtype):
    """Rows where a selection can go wrong, V = 20 000."""
    V = 20_000
    low = torch.finfo(dtype).min
    g = torch.Generator().manual_seed(5)
    x = torch.randn(19, V, generator=g).to(dtype)
    x[0] = 1.5                                        # all alike: the first words
    x[1] = torch.arange(V).to(dtype)                  # ascending
    x[2] = -torch.arange(V).to(dtype)                 # descending
    x[3] = -INF                                       # masked whole
    x[4, 5:] = -INF                                   # fewer words than places
    x[5] = low                                        # all at the type's lowest value
    x[6, 100:] = low
    x[7, ::2] = -INF
    x[8] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)      # zeros of both signs are alike
    x[9, 777] = NAN
    x[9, 12] = -NAN
    x[10, [3, 19_999]] = INF
    x[11, 19_999] = 50.0
    x[12] = (torch.arange(V) // 100 % 7).to(dtype)    # long ties
    x[13, :4000] = 9.0                                # more ties at the top than a list holds
    x[14] = torch.finfo(dtype).max
    x[15] = -INF
    x[15, 19_000:19_300] = 2.0
    x[16, :] = -INF
    x[16, 7] = NAN
    x[17, 5000:5600] += 20                            # the largest words next to each other
    x[18] *= 1e-6 if dtype == F32 else 1.0
    return x.cuda()


@pytest.mark.parametrize("top", [1, 20, 64, 300, 512])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_top_logits_where_a_selection_can_go_wrong(dtype, top):
    check_top(special_rows(dtype), top)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_top_logits_where_a_selection_can_go_wrong_in_many_rows(dtype):
    """The same rows among so many that each has one CTA."""
    x = special_rows(dtype)
    few = rows.top_logits(x, 100)
    check_top(x, 100)
    many = rows.top_logits(x.repeat(64, 1), 100)
    for a, c in zip(few[:2], many[:2]):
        c = c.view(64, *a.shape)
        a, c = torch.nan_to_num(a.float(), nan=1.0, posinf=2.0, neginf=3.0), torch.nan_to_num(c.float(), nan=1.0, posinf=2.0, neginf=3.0)
        assert bool((c == a).all())
    bound = 2 * (lse_error(x.cpu().double(), 1.0) + 2.0**-23 + HALF_STEP[F32] * few[2].cpu().double().abs())
    off = (many[2].view(64, -1) - few[2]).abs().cpu().double()
    plain = torch.isfinite(few[2]).cpu()
    assert bool((off <= bound)[:, plain].all())
    assert torch.equal(torch.nan_to_num(many[2].view(64, -1)[:, ~plain], nan=5.0), torch.nan_to_num(few[2][~plain], nan=5.0).expand(64, -1))


@pytest.mark.parametrize("top", [5, 64, 301])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_top_logits_at_borders_of_any_size_and_sign(dtype, top):
    # values around the border: of both signs next to zero (16-bit rows: subnormal numbers and both zeros), and of one sign over all
    # exponents up to 2^14
    V = 20011
    g = torch.Generator().manual_seed(41)
    bits = torch.randint(0, 1 << 10, (4, V), generator=g) - torch.randint(0, 2, (4, V), generator=g) * (1 << 15)
    tiny = bits.to(torch.int16).view(F16 if dtype is F16 else BF16).to(dtype)
    wide = torch.exp2(torch.rand(4, V, generator=g, dtype=torch.float64) * 38 - 24).to(dtype)
    wide[2:] = -wide[2:]
    wide[1::2, ::3] = -INF
    check_top(torch.cat([tiny, wide]).cuda(), top)


def test_top_logits_of_one_row_again_and_again():
    x = make(1, 5_003, BF16, 1).expand(6, 5_003)       # row stride 0
    check_top(x, 9)


# --- distillation ------------------------------------------------------------------------------------------------------------

def distill_reference(x, ids, values, lse, tau, weights):
    """Loss and gradient in 64 bits on the CPU, each with a bound of the kernels' error (module docstring, and below)."""
    n, V = x.shape
    x = x.double()
    loss, loss_tol = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    grad, grad_tol = torch.zeros(n, V, dtype=torch.float64), torch.zeros(n, V, dtype=torch.float64)
    sums = lse_error(x, tau)
    for r in range(n):
        at = [j for j in range(ids.shape[1]) if 0 <= int(ids[r, j]) < V]
        if not at:
            continue
        words = ids[r, at].long()
        t = values[r, at].double() / tau
        a = t - lse[r].double() if lse is not None else torch.log_softmax(t, 0) if bool((t > -INF).any()) else t
        p = torch.exp(a)
        y = x[r] / tau
        log_q = torch.log_softmax(y, 0) if not bool((y == -INF).all()) else y
        q = torch.exp(log_q)
        out = torch.ones(V, dtype=torch.bool)
        out[words] = False
        q_rest = q[out].sum()
        p_rest = torch.clamp(1 - p.sum(), min=0) if lse is not None and q_rest > 0 else torch.zeros((), dtype=torch.float64)
        ratio = torch.where(p > 0, a - log_q[words], 0.0)
        rest_ratio = torch.log(p_rest / q_rest) if p_rest > 0 else torch.zeros((), dtype=torch.float64)
        loss[r] = tau**2 * ((p * ratio).sum() + p_rest * rest_ratio)
        # p: the argument of the exponential is rounded once, expf is 2 units off; renormalised lists divide by such a sum
        ep = 2.0**-22 + 2.0**-24 * (torch.where(p > 0, a.abs(), 0.0).max()) + (2.0**-21 if lse is None else 0.0)
        es = sums[r] + 2.0**-22
        total_p = p.sum()
        loss_tol[r] = tau**2 * (es * (total_p + p_rest) + ep * ((p * ratio.abs()).sum() + total_p * (1 + rest_ratio.abs()))
                                + (p_rest * es if p_rest > 0 else 0.0))
        loss_tol[r] += HALF_STEP[F32] * loss[r].abs()
        w = float(weights[r]) * tau
        mass = total_p + p_rest
        g = q * mass
        g.index_add_(0, words, -p)
        # e of one word: the argument's roundings, 2^-22; three products in single precision
        eq = 2.0**-22 + 3 * 2.0**-24 * torch.nan_to_num((y.max() - y) * 1.4427, nan=0.0, posinf=0.0) + es + 4 * 2.0**-24
        tol = (q + 2.0**-126) * mass * eq + 2.0**-126 * mass + q * ep * total_p
        tol.index_add_(0, words, p * ep)
        if p_rest > 0:
            g[out] -= p_rest * q[out] / q_rest
            tol[out] += ((q[out] + 2.0**-126) * (p_rest * (eq[out] + es) + ep * total_p) + 2.0**-126 * p_rest) / q_rest
        grad[r], grad_tol[r] = g * w, tol * abs(w)
        if w == 0:
            grad[r] = grad_tol[r] = 0.0
    return loss, loss_tol, grad, grad_tol


def lists_of(teacher, top, tau, tail, dtype):
    """A teacher's lists by the plain reference (CPU), as the operator's inputs."""
    ids, values, lse = top_reference(teacher, top, tau)
    return ids.cuda(), values.to(dtype).cuda(), lse.float().cuda() if tail else None


def same(got, want, tol, dtype):
    got = got.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    odd = ~torch.isfinite(want)
    assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)])
    off = (got - want).abs()[~odd]
    bound = (tol + HALF_STEP[dtype] * (want.abs() + tol) + SMALLEST[dtype])[~odd]
    assert bool((off <= bound).all()), (float((off - bound).max()), int((off > bound).sum()))


def check_distill(x, ids, values, lse, tau=1.0, weights=None, in_place=False):
    n = x.shape[0]
    w = torch.ones(n) if weights is None else weights.cpu()
    want_loss, loss_tol, want_grad, grad_tol = distill_reference(x.cpu(), ids.cpu(), values.cpu(),
                                                                 None if lse is None else lse.cpu(), tau, w)
    alone = rows.distill_loss(x, ids, values, lse, temperature=tau)
    same(alone, want_loss, loss_tol, F32)
    loss, grad = rows.distill_loss_and_grad(x, ids, values, lse, temperature=tau, weights=weights, grad=x if in_place else None)
    same(loss, want_loss, loss_tol, F32)
    same(grad, want_grad, grad_tol, x.dtype)
    return loss, grad


DISTILL_SIZES = [(1, 1, 1), (2, 1, 3), (3, 2, 1), (3, 7, 7), (2, 33, 8), (4, 300, 64), (3, 1000, 512), (17, 1_009, 12), (2, 4_099, 33),
                 (150, 515, 9), (601, 257, 5), (3, 50_021, 100), (2, 141_000, 64), (1, 1_000_000, 40), (1, 1 << 20, 512)]


@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("n_rows,V,top", DISTILL_SIZES)
def test_distill(n_rows, V, top, dtype, tail):
    x = make(n_rows, V, dtype, seed=V)
    ids, values, lse = lists_of(make(n_rows, V, dtype, seed=V + 1).cpu(), top, 2.0, tail, dtype)
    check_distill(x, ids, values, lse, tau=2.0)


@pytest.mark.parametrize("values_dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_distill_lists_of_another_type(dtype, values_dtype):
    x = make(3, 2_000, dtype, 1)
    ids, values, lse = lists_of(make(3, 2_000, F32, 2).cpu(), 50, 1.0, True, values_dtype)
    check_distill(x, ids, values, lse)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 3), (5, 1), (8, 8), (16, 4)])
def test_distill_rows_at_any_address(dtype, pad, offset):
    V = 3_331
    x = make(5, V, dtype, 3, pad, offset=offset)
    ids, values, lse = lists_of(make(5, V, dtype, 4).cpu(), 21, 0.7, True, dtype)
    w = torch.tensor([0.5, -2.0, 0.0, 1.0, 3.0], device="cuda")
    before = x.clone()
    # the gradient's rows lie elsewhere than the logits', at another offset from 16 bytes
    flat = torch.full((7 + 5 * (V + 2),), 55.0, dtype=dtype, device="cuda")
    grad = flat[7:].view(5, V + 2)[:, :V]
    loss, got = rows.distill_loss_and_grad(x, ids, values, lse, temperature=0.7, weights=w, grad=grad)
    assert got is grad and torch.equal(x, before)
    assert bool((flat[:7] == 55).all()) and bool((flat[7:].view(5, V + 2)[:, V:] == 55).all())      # nothing between the rows
    _, fresh = check_distill(x, ids, values, lse, tau=0.7, weights=w)
    assert torch.equal(fresh, grad)
    check_distill(x, ids, values, lse, tau=0.7, weights=w, in_place=True)
    assert torch.equal(x, fresh)
    whole = x.as_strided((5, V + pad), (V + pad, 1))
    assert bool((whole[:4, V:] == 77).all())


def test_distill_long_lists_strided_lists_and_padding():
    V = 5_000
    x = make(6, V, BF16, 8)
    ids, values, lse = lists_of(make(6, V, BF16, 9).cpu(), 128, 1.0, True, BF16)
    ids = ids.clone()
    ids[1, 40:] = -1
    ids[2, ::2] = V                                    # outside the vocabulary: padding as well
    ids[3] = -7                                        # nothing but padding
    ids[4, 1:] = 2**31 - 1
    ids[5, 3] = -2**31
    loss, grad = check_distill(x, ids, values, lse)
    assert float(loss[3]) == 0.0 and bool((grad[3] == 0).all())
    check_distill(x, ids, values, None)
    check_distill(x, ids[:, :33], values[:, :33], lse)              # list stride 128
    check_distill(x[:1], ids[:1], values[:1], lse[:1])


def test_distill_a_word_listed_twice():
    V = 700
    x = make(4, V, F32, 8)
    ids, values, lse = lists_of(make(4, V, F32, 9).cpu(), 16, 1.0, True, F32)
    lse = lse + 1.0                                     # both entries count, and their sum stays below one
    ids = ids.clone()
    ids[0, 5] = ids[0, 4]
    ids[1, :] = 17
    ids[2, [3, 9, 15]] = ids[2, 0].item()
    first = check_distill(x, ids, values, lse)
    second = rows.distill_loss_and_grad(x, ids, values, lse)
    assert torch.equal(first[1], second[1])
    check_distill(x, ids, values, None)


@pytest.mark.parametrize("n_rows", [10, 1300])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
def test_distill_masked_and_infinite_places(dtype, tail, n_rows):
    """A few rows are shared out over clusters, many have one CTA each."""
    V, low = 6_000, torch.finfo(dtype).min
    x = make(10, V, dtype, 11)
    teacher = make(10, V, dtype, 12)
    teacher[0, 100:] = -INF
    x[0, 100:] = -INF                                   # both masked: nothing outside a list of 100
    x[1, ::3] = -INF                                    # some listed words have no mass: infinite loss where the teacher has some
    x[2] = -INF                                         # the student is masked whole
    x[3] = low                                          # all at the type's lowest value: uniform
    x[4, 64:] = low
    teacher[5] = low
    x[6, 10] = NAN
    x[8] = 0
    x[9] *= 8
    ids, values, lse = lists_of(teacher.cpu(), 100, 1.0, tail, dtype)
    values = values.clone()
    values[7, 3] = NAN
    w = torch.full((10,), 2.0, device="cuda")
    if n_rows > 10:
        again = lambda t: t.repeat(n_rows // 10, *[1] * (t.dim() - 1))      # noqa: E731
        want_loss, loss_tol, want_grad, grad_tol = distill_reference(x.cpu(), ids.cpu(), values.cpu(), None if lse is None else lse.cpu(), 1.0, w.cpu())
        loss, grad = rows.distill_loss_and_grad(again(x), again(ids), again(values), None if lse is None else again(lse), weights=again(w))
        alone = rows.distill_loss(again(x), again(ids), again(values), None if lse is None else again(lse))
        for k in (0, n_rows // 20, n_rows // 10 - 1):
            same(loss[10 * k: 10 * k + 10], want_loss, loss_tol, F32)
            same(alone[10 * k: 10 * k + 10], want_loss, loss_tol, F32)
            same(grad[10 * k: 10 * k + 10], want_grad, grad_tol, dtype)
        return
    loss, grad = check_distill(x, ids, values, lse, weights=w)
    assert math.isinf(float(loss[2])) and bool(torch.isfinite(grad[2]).all())
    assert bool(torch.isnan(grad[6]).all()) and bool(torch.isnan(loss[6])) and bool(torch.isnan(loss[7]))
    # a row of weight 0 passes nothing on, whatever it holds
    w[6] = w[7] = w[2] = 0.0
    _, grad = rows.distill_loss_and_grad(x, ids, values, lse, weights=w)
    assert bool((grad[[2, 6, 7]] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("above", [60.0, 100.0, 300.0])
def test_distill_student_with_next_to_no_mass_outside_the_list(dtype, above):
    """The words outside the list have e^-above of the student's mass, less than a single-precision number holds: their gradient
    is -tau P share, share their softmax among themselves.  Errors: those of the sums and of one exponential, P's is 2^-22."""
    V, top, tau = 5_000, 40, 1.0
    x = make(3, V, dtype, 61)
    ids, values, lse = lists_of(make(3, V, dtype, 62).cpu(), top, tau, True, dtype)
    lse = lse + 0.5                                     # the teacher has more mass outside
    x.scatter_add_(1, ids.long(), torch.full((3, top), above, dtype=dtype, device="cuda"))
    loss, grad = rows.distill_loss_and_grad(x, ids, values, lse, temperature=tau)
    d = x.cpu().double()
    outside = torch.ones(3, V, dtype=torch.bool).scatter_(1, ids.cpu().long(), False)
    rest = d.masked_fill(~outside, -INF)
    p = torch.exp(values.cpu().double() / tau - lse.cpu().double()[:, None])
    p_rest = 1 - p.sum(1)
    log_p = values.cpu().double() / tau - lse.cpu().double()[:, None]
    log_q = torch.gather(torch.log_softmax(d / tau, 1), 1, ids.cpu().long())
    log_q_rest = torch.logsumexp(rest / tau, 1) - torch.logsumexp(d / tau, 1)
    want = tau**2 * ((p * (log_p - log_q)).sum(1) + p_rest * (torch.log(p_rest) - log_q_rest))
    assert bool(((loss.cpu().double() - want).abs() <= 2e-5 * tau**2 + 2.0**-22 * (want.abs() + above)).all())
    share = torch.softmax(rest / tau, 1)
    far = torch.nan_to_num((rest.max(1, keepdim=True).values - rest) / tau, posinf=0.0)
    want = -tau * p_rest[:, None] * share + tau * torch.softmax(d / tau, 1).masked_fill(~outside, 0.0)
    got = grad.cpu().double().masked_fill(~outside, 0.0)
    error = DEPTH * 2.0**-23 + 2.0**-20 + 3 * 2.0**-24 * far * 1.4427 + 2.0**-22 / p_rest[:, None]
    bound = want.abs() * (error + HALF_STEP[dtype]) + tau * 2.0**-24 * share + SMALLEST[dtype] + 2.0**-126
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())


def test_distill_teacher_without_mass_on_its_list():
    x = make(2, 400, F32, 1)
    ids, values, lse = lists_of(make(2, 400, F32, 2).cpu(), 10, 1.0, True, F32)
    values = torch.full_like(values, -INF)
    check_distill(x, ids, values, lse)                  # all of it is outside the list
    loss, grad = check_distill(x, ids, values, None)    # none at all
    assert bool((loss == 0).all()) and bool((grad == 0).all())


@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
def test_distill_gradient_against_differences(tail):
    """Along a direction with entries of -1 and 1: |third derivative| of a log-sum-exp is at most 8 / tau^3 there, the loss holds
    tau^2 (W lse + P lse') of them with W, P <= 1, and each loss is off by loss_tol at most."""
    V, tau, h = 3_001, 1.5, 2.0**-4
    x = make(8, V, F32, 21)
    ids, values, lse = lists_of(make(8, V, F32, 22).cpu(), 40, tau, tail, F32)
    d = (torch.randint(0, 2, (8, V), generator=torch.Generator().manual_seed(3)) * 2 - 1).float().cuda()
    _, grad = rows.distill_loss_and_grad(x, ids, values, lse, temperature=tau)
    _, loss_tol, _, grad_tol = distill_reference(x.cpu(), ids.cpu(), values.cpu(), None if lse is None else lse.cpu(), tau, torch.ones(8))
    up = rows.distill_loss(x + h * d, ids, values, lse, temperature=tau).double()
    down = rows.distill_loss(x - h * d, ids, values, lse, temperature=tau).double()
    slope = (grad.double() * d).sum(1)
    # (x + h d is rounded as well: by 2^-24 |x| per word, which moves the loss by at most the sum of |gradient| 2^-24 |x|)
    moved = (grad.abs().double() * (x.abs() + 1) * 2.0**-24).sum(1).cpu() / h
    bound = (2 * loss_tol + 1e-7) / h + h * h / 6 * 16 / tau + moved + grad_tol.sum(1)
    assert bool((((up - down) / (2 * h) - slope).abs().cpu() <= bound).all())
    assert float(slope.abs().max()) > 4 * float(bound.max())      # the bound says something


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_distill_through_autograd(dtype):
    V = 2_003
    x = make(5, V, dtype, 31).clone().requires_grad_()
    ids, values, lse = lists_of(make(5, V, dtype, 32).cpu(), 24, 1.0, True, dtype)
    w = torch.tensor([1.0, 0.0, 2.0, -1.0, 0.25], device="cuda")
    loss = rows.distill_loss(x, ids, values, lse)
    (loss * w).sum().backward()
    plain_loss, plain = rows.distill_loss_and_grad(x, ids, values, lse, weights=w)
    assert torch.equal(loss, plain_loss) and torch.equal(x.grad, plain) and not plain.requires_grad
    # a broadcast student: its gradient is the rows' sum; a mean's gradient arrives with stride 0
    one = x[:1].detach().clone().requires_grad_()
    rows.distill_loss(one.expand(5, V), ids, values, lse).mean().backward()
    each = rows.distill_loss_and_grad(one.detach().expand(5, V), ids, values, lse, weights=torch.full((5,), 0.2, device="cuda"))[1]
    want = each.sum(0, keepdim=True)
    assert bool(((one.grad - want).abs() <= 5 * 2 * HALF_STEP[dtype] * each.abs().sum(0)).all())
    with torch.no_grad():
        assert not rows.distill_loss(x, ids, values, lse).requires_grad
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(rows.distill_loss(x, ids, values, lse).sum(), x, create_graph=True)
        g.sum().backward()


# --- a list far above or far below the words outside it -----------------------------------------------------------------------

def check_apart(x, ids, values, lse, tau):
    """Loss and gradient where the list and the words outside it lie any distance apart: all in logarithms, in 64 bits.

    Errors.  log q: the exponents' factor c is rounded (2^-24 of |log q|, and as much of the distance between the two sums, which
    counts by their share: 2^-24 of at most 1), both sums are `s` off, each by its own largest word.  p: ep as above, its logarithm
    2^-24 |log p|; P is as far off as the sum of the p.  Gradient: one exponential more, relative to the largest on its side, or 0 below 2^-126."""
    n, V = x.shape
    d, at = x.cpu().double(), ids.cpu().long()
    outside = torch.ones(n, V, dtype=torch.bool).scatter_(1, at, False)
    listed, rest = torch.gather(d, 1, at) / tau, d.masked_fill(~outside, -INF) / tau
    log_in, log_out = torch.logsumexp(listed, 1, keepdim=True), torch.logsumexp(rest, 1, keepdim=True)
    log_z = torch.logaddexp(log_in, log_out)
    a = values.cpu().double() / tau - lse.cpu().double()[:, None]
    p = torch.exp(a)
    p_rest = 1 - p.sum(1, keepdim=True)
    assert float(p_rest.min()) > 0.1
    log_q, log_q_rest = listed - log_z, log_out - log_z
    ratio, rest_ratio = a - log_q, torch.log(p_rest) - log_q_rest
    want_loss = tau**2 * ((p * ratio).sum(1) + (p_rest * rest_ratio)[:, 0])
    s = torch.maximum(lse_error(listed * tau, tau), lse_error(rest * tau, tau))[:, None] + 2.0**-24
    ep = 2.0**-22 + 2.0**-24 * a.abs().max(1, keepdim=True).values
    off_p = ep * p.sum(1, keepdim=True)
    loss_tol = (p * (2.0**-24 * (log_q.abs() + a.abs()) + s + ep * ratio.abs())).sum(1, keepdim=True) \
        + p_rest * (2.0**-24 * log_q_rest.abs() + 2 * s) + off_p * (rest_ratio.abs() + 1)
    loss_tol = tau**2 * loss_tol[:, 0]
    mass = p.sum(1, keepdim=True) + p_rest
    apart = torch.clamp((log_z - log_out) * 1.4427 * 2.0**-24, max=1.0)      # of e^(log_out - log_z)

    def one(y):      # a word's exponential, by its distance from the largest on its side
        return 2.0**-22 + 3 * 2.0**-24 * torch.nan_to_num((y.max(1, keepdim=True).values - y) * 1.4427, posinf=0.0) + 8 * 2.0**-24
    share = torch.softmax(rest, 1)      # (by differences of the logits: at the lowest values a logarithm has no places for their number)
    q = share * torch.exp(log_out - log_z)
    want = mass * q - p_rest * share
    tol = (mass * q + p_rest * share) * (one(rest) + 2 * s) + mass * q * apart + share * off_p + 2.0**-126 * mass
    q_list = torch.softmax(listed, 1) * torch.exp(log_in - log_z)
    tol_list = mass * q_list * (one(listed) + 2 * s + torch.clamp((log_z - log_in) * 1.4427 * 2.0**-24, max=1.0)) \
        + q_list * off_p + p * ep + 2.0**-126 * mass
    want.scatter_(1, at, mass * q_list - p)
    tol.scatter_(1, at, tol_list)
    many = 1500 // n      # a CTA each
    for times in (1, many):
        again = [t.repeat(times, *[1] * (t.dim() - 1)) for t in (x, ids, values, lse)]
        alone = rows.distill_loss(*again, temperature=tau)
        loss, grad = rows.distill_loss_and_grad(*again, temperature=tau)
        for part in (slice(0, n), slice((times - 1) * n, times * n)):
            same(alone[part], want_loss, loss_tol, F32)
            same(loss[part], want_loss, loss_tol, F32)
            same(grad[part], tau * want, tau * tol, x.dtype)


def apart(V, dtype, seed, tau, spread=3.0):
    """Three rows of ordinary logits, in units of tau, and a teacher's lists of 40 with four tenths of its mass outside."""
    x = (make(3, V, F32, seed, spread=spread) * tau).to(dtype)
    ids, values, lse = lists_of((make(3, V, F32, seed + 1) * tau).to(dtype).cpu(), 40, tau, True, dtype)
    p = torch.exp(values.double() / tau - lse.double()[:, None]).sum(1)
    return x, ids, values, (lse.double() + torch.log(p / 0.6)).float()


@pytest.mark.parametrize("V", [5_000, 40_000])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("tau,above", [(1.0, 600.0), (1.0, 800.0), (1.0, 1000.0), (1.0, 20_000.0), (0.01, 7.5), (0.01, 12.0), (30.0, 30_000.0)])
def test_distill_list_far_above_the_words_outside(tau, above, dtype, V):
    x, ids, values, lse = apart(V, dtype, 71, tau)
    x.scatter_add_(1, ids.long(), torch.full((3, 40), above, dtype=dtype, device="cuda"))
    check_apart(x, ids, values, lse, tau)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("low", [-1e4, -6e4])
def test_distill_words_outside_the_list_at_a_low_value(low, dtype):
    x, ids, values, lse = apart(6_000, dtype, 73, 1.0)
    x = torch.full_like(x, low).scatter_(1, ids.long(), torch.gather(x, 1, ids.long()))
    check_apart(x, ids, values, lse, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("above", [20.0, 41.0, 55.0, 64.0, 67.0, 68.5, 69.5, 75.0, 86.0])
def test_distill_gradient_of_words_far_below_the_list(above, dtype):
    """Words outside the list lie up to 50 below the largest of them, which itself lies `above` below the list."""
    x, ids, values, lse = apart(5_000, dtype, 75, 1.0, spread=6.0)
    x.scatter_(1, ids.long(), x.max(1, keepdim=True).values.expand(3, 40) + above)
    check_apart(x, ids, values, lse, 1.0)


@pytest.mark.parametrize("above", [0.0, 100.0, 150.0, 2000.0, -40.0, -150.0, -2000.0])
@pytest.mark.parametrize("base", [0.0, 3000.0, -3000.0, 2.0**15])
def test_distill_does_not_depend_on_a_constant_added_to_the_row(base, above):
    """At this temperature rows that lie 3000 from zero have exponents beyond 2^22 (2^15: beyond 2^25).  All sums are exact."""
    tau, V = 1e-3, 40_000
    x, ids, values, lse = apart(V, F32, 77, tau)
    x = torch.round(x * 2.0**8) / 2.0**8               # (with the base, at most 24 bits)
    x.scatter_add_(1, ids.long(), torch.full((3, 40), round(above * tau * 2**8) / 2**8, device="cuda"))
    check_apart(x + base, ids, values, lse, tau)


@pytest.mark.parametrize("V", [5_000, 40_000])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("side", ["outside", "list"])
def test_distill_one_side_at_the_lowest_value(side, dtype, V):
    """Words at the type's lowest value are words: only minus infinity has no mass."""
    tau = 0.5                                           # (tau^2 times the lowest value is still a number)
    x, ids, values, lse = apart(V, dtype, 79, tau)
    at, low = ids.long(), torch.finfo(dtype).min
    if side == "outside":
        x = torch.full_like(x, low).scatter_(1, at, torch.gather(x, 1, at))
    else:
        x.scatter_(1, at, low)
    check_apart(x, ids, values, lse, tau)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
def test_distill_rows_far_from_zero_in_steps_of_their_type(dtype):
    tau = 1e-3
    x, ids, values, lse = apart(5_000, dtype, 81, 1.0)
    values, lse = values * tau, lse * 1.0
    values = (values.float()).to(F32)
    p = torch.exp(values.double() / tau - lse.double()[:, None]).sum(1)
    lse = (lse.double() + torch.log(p / 0.6)).float()
    steps = torch.randint(0, 4, (3, 5_000), generator=torch.Generator().manual_seed(5)).cuda()
    x = (2944 + 16 * steps).to(dtype)                  # 23 000 powers of two from one to the next
    check_apart(x, ids, values, lse, tau)


@pytest.mark.parametrize("top", [300, 512, 37])
@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
def test_distill_student_that_has_learnt_its_teacher(tail, top):
    """All words alike on both sides: the student's exponentials and sums are exact, and so are the list's e^0; what is left is the
    logarithms', in 64 bits.  With a tail p is expf's, two units of the last place off at most (2^-22), and P by as much the other way:
    with both ratios next to 1 the loss moves by that, its own derivative, and by its square."""
    V = top if not tail else 2 * top
    x = torch.zeros(2, V, device="cuda")
    ids = torch.arange(top, dtype=torch.int32, device="cuda").repeat(2, 1)
    values = torch.zeros(2, top, device="cuda")
    lse = torch.full((2,), math.log(V), device="cuda") if tail else None
    want, bound = 0.0, 1e-12
    if tail:
        a = -float(lse[0])
        p = top * math.exp(a)
        want = p * (a + math.log(V)) + (1 - p) * (math.log(1 - p) + math.log(2))
        bound += p * 2.0**-22 * (1 + 2.0**-20)
    got = rows.distill_loss(x, ids, values, lse).cpu().double()
    assert bool(((got - want).abs() <= bound + 2.0**-24 * abs(want)).all()), (got, want)


@pytest.mark.parametrize("tau", [0.5, 1e-3, 2.0])
@pytest.mark.parametrize("values_dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("tail", [False, True], ids=["list", "tail"])
def test_distill_teacher_with_words_at_the_lowest_value(tail, values_dtype, tau):
    """Some places of the list, or (without a tail) all of one, at the lowest value: t / tau is beyond single precision then."""
    x = make(3, 2_000, F32, 83)
    ids, values, lse = lists_of(make(3, 2_000, F32, 84, spread=3.0 * min(tau, 1.0)).cpu(), 40, tau, tail, values_dtype)
    values = values.clone()
    values[0, 20:] = torch.finfo(values_dtype).min
    values[1, ::2] = torch.finfo(values_dtype).min
    if not tail:
        values[2] = torch.finfo(values_dtype).min
    check_distill(x, ids, values, lse, tau=tau)


# --- verification of drafts --------------------------------------------------------------------------------------------------

def verify_reference(offsets, drafts, target, probs, au, du):
    """The definition with Python's whole numbers and exact products (a float's product of two floats is exact in 64 bits)."""
    offsets, drafts, au, du = offsets.tolist(), drafts.tolist(), au.tolist(), du.tolist()
    target = target.cpu().float()
    probs = None if probs is None else probs.cpu().float()
    V, n = target.shape[1], len(offsets) - 1
    tokens, accepted = [-1] * (len(drafts) + n), []
    for s in range(n):
        i, hi = offsets[s], offsets[s + 1]
        while i < hi and 0 <= drafts[i] < V:
            q = 1.0 if probs is None else float(probs[i, drafts[i]])
            if not au[i] * q < float(target[i + s, drafts[i]]):
                break
            tokens[i + s] = drafts[i]
            i += 1
        accepted.append(i - offsets[s])
        p = target[i + s]
        r = p.clone()
        if i < hi and probs is not None:
            r = p - probs[i]
        elif i < hi and 0 <= drafts[i] < V:
            r[drafts[i]] = 0
        u = du[s]
        U = 0 if not u > 0 else 2**32 - 1 if u >= 1 else int(u * 2**32)
        for row in (r, p):
            mass = torch.floor(torch.nan_to_num(row, nan=0.0).clamp(0, 1).double() * 2.0**42).to(torch.int64)
            total = int(mass.sum())
            if total:
                want = total * U >> 32
                tokens[i + s] = int(torch.searchsorted(torch.cumsum(mass, 0), want, right=True))
                break
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(accepted, dtype=torch.int32)


def drafts_of(lengths, V, dtype, seed, pad=0, one_hot=False, near=0.5, offset=0):
    g = torch.Generator().manual_seed(seed)
    n, total = len(lengths), sum(lengths)
    offsets = torch.tensor([0] + lengths).cumsum(0)
    seq = torch.repeat_interleave(torch.arange(n), torch.tensor(lengths, dtype=torch.int64))
    x = torch.randn(total + n, V, generator=g) * 3
    p = torch.softmax(x, 1).to(dtype)
    q = torch.softmax(x[torch.arange(total) + seq] + near * torch.randn(total, V, generator=g), 1).to(dtype)
    drafts = torch.multinomial(q.float(), 1, generator=g)[:, 0].to(torch.int32) if total and V <= 1 << 20 else torch.zeros(total, dtype=torch.int32)
    if V > 100_000:
        drafts = torch.where(torch.rand(total, generator=g) < 0.8, p[torch.arange(total) + seq].float().argmax(1).to(torch.int32), drafts)

    def lay(m):
        flat = torch.full((offset + m.shape[0] * (V + pad),), 9.0, dtype=dtype, device="cuda")
        view = flat[offset:].view(m.shape[0], V + pad)[:, :V]
        view.copy_(m)
        return view
    return (offsets.cuda(), drafts.cuda(), lay(p), None if one_hot else lay(q), torch.rand(total, generator=g).cuda(),
            torch.rand(n, generator=g).cuda())


def check_verify(args):
    tokens, accepted = rows.verify_drafts(*args)
    want_tokens, want_accepted = verify_reference(*args)
    assert torch.equal(accepted.cpu(), want_accepted)
    assert torch.equal(tokens.cpu(), want_tokens)
    return tokens, accepted


VERIFY_SIZES = [([0], 1), ([1], 1), ([3], 2), ([4, 0, 2], 7), ([1] * 5, 32), ([5, 3, 0, 8], 1_000), ([4], 10_000), ([2, 7, 1, 0, 3], 4_099),
                ([3] * 40, 515), ([i % 4 for i in range(200)], 257), ([2, 3], 50_021), ([4, 1, 3], 131_072), ([2], 1_000_000),
                ([1, 2], 1 << 20), ([300, 0, 257], 64)]


@pytest.mark.parametrize("one_hot", [False, True], ids=["probs", "lookup"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("lengths,V", VERIFY_SIZES, ids=lambda x: str(x)[:20])
def test_verify(lengths, V, dtype, one_hot):
    check_verify(drafts_of(lengths, V, dtype, V + len(lengths), one_hot=one_hot, near=0.02 if len(lengths) == 3 and V == 64 else 0.5))


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (3, 2), (8, 8), (4, 4)])
def test_verify_rows_at_any_address(dtype, pad, offset):
    check_verify(drafts_of([3, 0, 5, 1], 5_001, dtype, 1, pad=pad, offset=offset))


@pytest.mark.parametrize("u", [0.0, 2.0**-33, 0.5, 1 - 2.0**-24, 1.0, 7.0, -1.0, NAN])
def test_verify_random_numbers_at_their_limits(u):
    args = list(drafts_of([2, 0, 4], 900, F32, 2))
    args[5] = torch.full_like(args[5], u)
    check_verify(args)
    args[4] = torch.full_like(args[4], u)
    check_verify(args)


@pytest.mark.parametrize("one_hot", [False, True], ids=["probs", "lookup"])
@pytest.mark.parametrize("V", [900, 40_007])
def test_verify_rows_without_mass_and_odd_values(V, one_hot):
    offsets, drafts, p, q, au, du = drafts_of([2] * 10, V, F32, 4, one_hot=one_hot)
    rows_of = lambda s: [2 * s + s, 2 * s + s + 1, 2 * s + s + 2]      # noqa: E731  target rows of sequence s
    p[rows_of(0)] = 0.0                                 # nothing can be drawn: -1
    p[rows_of(1)] = NAN
    p[rows_of(2)] = INF
    p[rows_of(3)] = -1.0
    if q is not None:
        q[8:10] = 1.0                                   # sequence 4: nothing left of p - q: p itself
        q[10:12] = p[rows_of(5)[:2]]                    # p = q: always accepted
        q[12:14] = NAN
        q[14:16] = 0.0
        au[8:10] = 0.9
    drafts[16] = -1                                     # no word of the vocabulary: refused, nothing taken out
    drafts[18] = V
    drafts[19] = 2**31 - 1
    p[rows_of(9)] = torch.tensor([0.0] * (V - 1) + [2.0**-42], device="cuda")
    tokens, accepted = check_verify((offsets, drafts, p, q, au, du))
    assert int(tokens[0]) == -1 and int(accepted[0]) == 0


def test_verify_leaves_places_of_no_sequence():
    args = drafts_of([3, 2], 500, BF16, 6)
    want_tokens, want_accepted = rows.verify_drafts(*args)
    # a batch padded to 9 drafts and 4 more rows behind the last sequence
    offsets, drafts, p, q, au, du = args
    more = lambda x, n, fill: torch.cat([x, torch.full((n, *x.shape[1:]), fill, dtype=x.dtype, device="cuda")])      # noqa: E731
    tokens = torch.full((11,), 123, dtype=torch.int32, device="cuda")
    got, acc = rows.verify_drafts(offsets, more(drafts, 4, -5), more(p, 4, NAN), more(q, 4, NAN), more(au, 4, NAN), du, tokens=tokens)
    assert got is tokens and torch.equal(got[:7], want_tokens) and bool((got[7:] == 123).all()) and torch.equal(acc, want_accepted)
    # offsets that run outside or downwards leave their sequence alone
    bad = torch.tensor([0, 10, 5, -1], device="cuda")
    tokens = torch.full((12,), 123, dtype=torch.int32, device="cuda")
    got, acc = rows.verify_drafts(bad, more(drafts, 4, -5), more(p, 5, 0.0), more(q, 4, 0.0), more(au, 4, 0.5),
                                  torch.rand(3, device="cuda"), tokens=tokens)
    assert acc.tolist() == [-1, -1, -1] and bool((got == 123).all())


def test_verify_follows_the_targets_distribution():
    """Accepted or drawn, the first token is distributed as p: 2^16 sequences of one draft, chi-square over 6 words.  The statistic
    exceeds 30 with probability 1.5e-5 (five degrees of freedom)."""
    n, V = 1 << 16, 6
    g = torch.Generator().manual_seed(9)
    p = torch.tensor([0.4, 0.25, 0.2, 0.1, 0.04, 0.01])
    q = torch.tensor([0.1, 0.2, 0.3, 0.3, 0.05, 0.05])
    drafts = torch.multinomial(q, n, replacement=True, generator=g).to(torch.int32).cuda()
    tokens, accepted = rows.verify_drafts(torch.arange(n + 1).cuda(), drafts, p.cuda().expand(2 * n, V), q.cuda().expand(n, V),
                                          torch.rand(n, generator=g).cuda(), torch.rand(n, generator=g).cuda())
    seen = torch.bincount(tokens[::2].cpu().long(), minlength=V).double()
    want = p.double() * n
    assert float(((seen - want) ** 2 / want).sum()) < 30
    share = float(torch.minimum(p, q).sum())
    assert abs(float(accepted.double().mean()) - share) < 5 * math.sqrt(share * (1 - share) / n)


# --- together, and how they are called ---------------------------------------------------------------------------------------

def test_lists_loss_and_verification_together():
    """A teacher's lists, a drafter that learns from them by plain descent, its drafts verified against the teacher."""
    V, n, tau = 1_000, 32, 1.0
    teacher = make(n, V, F32, 41)
    ids, values, lse = rows.top_logits(teacher, 64, temperature=tau)
    student = torch.zeros(n, V, device="cuda", requires_grad=True)
    for _ in range(3):
        loss = rows.distill_loss(student, ids, values, lse, temperature=tau)
        grad, = torch.autograd.grad(loss.sum(), student)
        same(grad, *distill_reference(student.detach().cpu(), ids.cpu(), values.cpu(), lse.cpu(), tau, torch.ones(n))[2:], F32)
        with torch.no_grad():
            student -= 20 * grad
    p = torch.softmax(teacher, 1)
    q = torch.softmax(student.detach(), 1)[: n - 8].contiguous()      # eight sequences of three drafts
    drafts = torch.multinomial(q, 1, generator=torch.Generator(device="cuda").manual_seed(1))[:, 0].to(torch.int32)
    offsets = torch.arange(0, 25, 3, device="cuda")
    g = torch.Generator().manual_seed(2)
    check_verify((offsets, drafts, p, q, torch.rand(24, generator=g).cuda(), torch.rand(8, generator=g).cuda()))


def all_results(x, ids, values, lse, w, args):
    """The operators' outputs, one after the other."""
    return (*rows.top_logits(x, 48), *rows.distill_loss_and_grad(x, ids, values, lse, weights=w),
            rows.distill_loss(x, ids, values, lse), *rows.verify_drafts(*args))


def inputs(seed, V=30_011, dtype=BF16):
    x = make(9, V, dtype, seed)
    ids, values, lse = lists_of(make(9, V, dtype, seed + 1).cpu(), 48, 1.0, True, dtype)
    w = torch.rand(9, generator=torch.Generator().manual_seed(seed)).cuda()
    return x, ids, values, lse, w, drafts_of([3, 0, 4], V, dtype, seed)


def test_calls_on_several_streams():
    ins = [inputs(s) for s in (1, 2, 3, 4)]
    want = [all_results(*i) for i in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    got = [[] for _ in ins]
    for _ in range(4):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(all_results(*ins[k]))
    torch.cuda.synchronize()
    for k, runs in enumerate(got):
        for run in runs:
            assert all(torch.equal(a, c) for a, c in zip(run, want[k]))


def test_two_captured_graphs_replayed_in_turn():
    ins = [inputs(s) for s in (5, 6)]
    fresh = [inputs(s) for s in (7, 8)]
    want = [[all_results(*i) for i in ins], [all_results(*i) for i in fresh]]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in ins:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(all_results(*i))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]

    def replay():
        torch.cuda.synchronize()
        for _ in range(3):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
    replay()
    for k in (0, 1):
        assert all(torch.equal(a, c) for a, c in zip(outs[k], want[0][k]))
    for i, f in zip(ins, fresh):                        # other inputs at the same addresses
        for a, c in zip(i[:5] + i[5], f[:5] + f[5]):
            if a.shape == c.shape:
                a.copy_(c)
    replay()
    for k in (0, 1):
        again = all_results(*ins[k])
        assert all(torch.equal(a, c) for a, c in zip(outs[k], again))


@pytest.mark.parametrize("through", ["autograd", "loss_and_grad"])
def test_a_captured_training_step(through):
    """Loss, gradient and a step of plain descent in one graph.  Without autograd an eager graph of the same tensor may live on (a
    captured backward pass of torch's breaks its capture then, whatever the operator)."""
    x, ids, values, lse, w, _ = inputs(9, V=5_003, dtype=F32)
    student = x.clone().requires_grad_()
    eager = rows.distill_loss(student, ids, values, lse) if through == "loss_and_grad" else None

    def step():
        if through == "autograd":
            loss = rows.distill_loss(student, ids, values, lse)
            grad, = torch.autograd.grad((loss * w).sum(), student)
            loss = loss.detach()
        else:
            loss, grad = rows.distill_loss_and_grad(student, ids, values, lse, weights=w)
        with torch.no_grad():
            student.sub_(grad, alpha=3.0)
        return loss, grad
    want = x.clone()
    for _ in range(5):
        loss, grad = rows.distill_loss_and_grad(want, ids, values, lse, weights=w)
        want.sub_(grad, alpha=3.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(4):
        graph.replay()
    assert torch.equal(student.detach(), want) and torch.equal(out[0], loss) and torch.equal(out[1], grad)
    assert eager is None or eager.requires_grad


def test_calls_from_compiled_functions():
    """The calls stay outside of a compiled function's graphs: other inputs, another stream, and a backward pass through them."""
    x, ids, values, lse, w, args = inputs(13, V=5_003, dtype=F32)
    top = torch.compile(lambda t: rows.top_logits(t * 1.0, 48), backend="eager")
    learn = torch.compile(lambda t: rows.distill_loss(t * 1.0, ids, values, lse), backend="eager")
    both = torch.compile(lambda t: rows.distill_loss_and_grad(t * 1.0, ids, values, lse, weights=w), backend="eager")
    verify = torch.compile(lambda p: rows.verify_drafts(args[0], args[1], p * 1.0, *args[3:]), backend="eager")
    for k in range(3):
        fresh = make(9, 5_003, F32, 14 + k)
        target = torch.softmax(make(10, 5_003, F32, 24 + k), 1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side if k else torch.cuda.current_stream()):
            got = (*top(fresh), learn(fresh), *both(fresh), *verify(target))
        torch.cuda.synchronize()
        want = (*rows.top_logits(fresh, 48), rows.distill_loss(fresh, ids, values, lse),
                *rows.distill_loss_and_grad(fresh, ids, values, lse, weights=w), *rows.verify_drafts(args[0], args[1], target, *args[3:]))
        assert all(torch.equal(a, c) for a, c in zip(got, want))
    student = x.clone().requires_grad_()
    (learn(student) * w).sum().backward()
    assert torch.equal(student.grad, rows.distill_loss_and_grad(x, ids, values, lse, weights=w)[1])


FIRST_IN_A_CAPTURE = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import torch
import test_gpu_rows as T
ins = T.inputs(3)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = T.all_results(*ins)
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(out, T.all_results(*ins)))
print("same")
"""


def test_the_first_calls_of_a_process_in_a_capture():
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", FIRST_IN_A_CAPTURE.format(root=os.path.dirname(here), tests=here)], capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]


def test_elements_beyond_32_bits():
    """Two rows 2^31 elements apart, and their gradient as far apart."""
    V, far = 40_009, (1 << 31) - 8
    flat = torch.empty(far + V, dtype=BF16, device="cuda")
    x = flat.as_strided((2, V), (far, 1))
    x.copy_(make(2, V, BF16, 51))
    check_top(x, 17)
    ids, values, lse = lists_of(make(2, V, BF16, 52).cpu(), 30, 1.0, True, BF16)
    out = torch.empty(far + V, dtype=BF16, device="cuda").as_strided((2, V), (far, 1))
    near = rows.distill_loss_and_grad(x.contiguous(), ids, values, lse)
    got = rows.distill_loss_and_grad(x, ids, values, lse, grad=out)
    assert torch.equal(got[0], near[0]) and torch.equal(got[1], near[1])
    args = drafts_of([1], V, BF16, 53)
    want = rows.verify_drafts(*args)
    x.copy_(args[2])
    got = rows.verify_drafts(args[0], args[1], x, *args[3:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_tensors_that_do_not_fit_are_refused():
    x = make(3, 50, F32, 1)
    ids, values, lse = lists_of(x.cpu(), 5, 1.0, True, F32)
    for bad in (x.double(), x.to(torch.int32)):
        with pytest.raises(TypeError):
            rows.top_logits(bad, 3)
    for bad in (x[0], x[:, ::2], x[:, :0], x.t()):
        with pytest.raises(ValueError):
            rows.top_logits(bad, 3)
    for top in (0, -1, b.LDA_TOP_MAX + 1):
        with pytest.raises(ValueError):
            rows.top_logits(x, top)
    with pytest.raises(b.LdaError):
        rows.top_logits(x, 3, temperature=0.0)
    with pytest.raises(TypeError):
        rows.distill_loss(x, ids.long(), values, lse)
    with pytest.raises(TypeError):
        rows.distill_loss(x, ids, values.double(), lse)
    with pytest.raises(TypeError):
        rows.distill_loss(x, ids, values, lse.double())
    for i, v, s in ((ids[:2], values, lse), (ids, values[:, :4], lse), (ids, values, lse[:2]), (ids[:, ::2], values[:, ::2], lse),
                    (ids[:, :0], values[:, :0], lse), (ids.cpu(), values, lse), (ids, values, lse.cpu()),
                    (ids, values.repeat(1, 2)[:, :5], lse)):
        with pytest.raises(ValueError):
            rows.distill_loss(x, i, v, s)
    with pytest.raises(ValueError):
        rows.distill_loss_and_grad(x, ids, values, lse, grad=torch.empty_like(x, dtype=BF16))
    with pytest.raises(ValueError):
        rows.distill_loss_and_grad(x, ids, values, lse, weights=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        rows.distill_loss_and_grad(x, ids, values, lse, grad=torch.empty_like(x).requires_grad_())
    with pytest.raises(b.LdaError):
        rows.distill_loss_and_grad(x, ids, values, lse, grad=torch.empty(50, device="cuda").expand(3, 50))
    offsets, drafts, p, q, au, du = drafts_of([2, 1], 50, F32, 1)
    for bad in ((offsets[:2], drafts, p, q, au, du), (offsets, drafts[:2], p, q, au, du), (offsets, drafts, p[:4], q, au, du),
                (offsets, drafts, p, q[:, :40], au, du), (offsets, drafts, p, q.half(), au, du), (offsets, drafts, p, q, au[:1], du),
                (offsets, drafts, p, q, au, du[:1]), (offsets.cpu(), drafts, p, q, au, du)):
        with pytest.raises(ValueError):
            rows.verify_drafts(*bad)
    for bad in ((offsets.int(), drafts, p, q, au, du), (offsets, drafts.long(), p, q, au, du), (offsets, drafts, p, q, au.double(), du)):
        with pytest.raises(TypeError):
            rows.verify_drafts(*bad)


def test_no_rows():
    x = torch.empty(0, 50, device="cuda")
    ids, values, lse = rows.top_logits(x, 4)
    assert ids.shape == values.shape == (0, 4) and lse.shape == (0,)
    loss, grad = rows.distill_loss_and_grad(x, ids, values, lse)
    assert loss.shape == (0,) and grad.shape == (0, 50)
    none = torch.empty(0, device="cuda")
    tokens, accepted = rows.verify_drafts(torch.zeros(1, dtype=torch.int64, device="cuda"), none.int(), x, x, none, none)
    assert tokens.shape == accepted.shape == (0,)
