"""The operators on a paged cache against plain forms in 64 bits.

Tolerances.  `HALF_STEP` is half the distance of neighbouring numbers, relative.  A rotated value is a sum of two products of single
precision with a cosine and a sine: three roundings of 2^-24, the functions' own error and that of the angle, which is worked out in 64 bits and
rounded once (2^-24 of pi at most), come to less than 2^-20 of |a| + |b|; then it is rounded once.

Attention: a score is a sum of `dim` products in single precision, off by at most (dim + 8) 2^-23 of the sum of their absolute values (a
matrix product may cut off where an addition rounds), so a probability is off by that, relative, and so is the norm; the exponential and its
argument add 2^-20 (arguments up to 2^2 of whole numbers, 2^-22 of the exponential itself); sums over `keys` terms in single precision keys 2^-24.
Probabilities are rounded to 16 bits before the product with the values: HALF_STEP of sum p |v|.  The output is rounded once.
"""
import math

import pytest
import torch

from paper_1412_1576_b200 import binding as b
from paper_1412_1576_b200 import cache, rows

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
HALF_STEP = {F16: 2.0**-11, BF16: 2.0**-8}
SMALLEST = {F16: 2.0**-25, BF16: 2.0**-134}
NAN, INF = float("nan"), float("inf")


class Batch:
    """Sequences with contexts `starts` and `new` tokens each, in a cache of random values."""

    def __init__(self, starts, new, kv_heads, dim, page, dtype, seed=0, by_head=False, extra_pages=3, behind=0, width=None):
        g = torch.Generator().manual_seed(seed)
        self.g, self.dtype, self.dim, self.page, self.kv_heads = g, dtype, dim, page, kv_heads
        n = len(new)
        self.starts = torch.tensor(starts, dtype=torch.int32).cuda()
        self.offsets = torch.tensor([sum(new[:i]) for i in range(n + 1)], dtype=torch.int64).cuda()
        self.tokens = sum(new) + behind
        need = [-(-(max(s, 0) + m) // page) for s, m in zip(starts, new)]
        pages = sum(need) + extra_pages
        order = torch.randperm(pages, generator=g).tolist()
        self.table = torch.full((n, width or max(need + [1])), -1, dtype=torch.int32)
        for i, k in enumerate(need):
            for j in range(min(k, self.table.shape[1])):
                self.table[i, j] = order.pop()
        self.table = self.table.cuda()
        shape = (pages, kv_heads, page, dim) if by_head else (pages, page, kv_heads, dim)
        self.k, self.v = (torch.randn(shape, generator=g).to(dtype).cuda() for _ in range(2))
        if by_head:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)

    def rows(self, heads, by=1.0):
        return (torch.randn(self.tokens, heads, self.dim, generator=self.g) * by).to(self.dtype).cuda()

    def where(self):
        return self.table, self.starts, self.offsets

    def slots(self, i):
        """Pages and places of a sequence's slots; -1 for no page."""
        lo, hi = self.offsets[i : i + 2].tolist()
        total = min(max(int(self.starts[i]), 0) + hi - lo, self.table.shape[1] * self.page)
        s = torch.arange(total, device="cuda")
        p = self.table[i].long()[s // self.page]
        return torch.where((p >= 0) & (p < self.k.shape[0]), p, -1), s % self.page


def attend_reference(x, q, mask=None, scale=None):
    """Outputs in 64 bits, and their tolerance; rows of no sequence are NaN."""
    heads, scale = q.shape[1], x.dim**-0.5 if scale is None else scale
    out = torch.full(q.shape, NAN, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    h = HALF_STEP[x.dtype]
    for i in range(x.offsets.numel() - 1):
        lo, hi = x.offsets[i : i + 2].tolist()
        n, start = hi - lo, max(int(x.starts[i]), 0)
        if n <= 0:
            continue
        pages, places = x.slots(i)
        k, v = (c[pages.clamp(min=0), places].double().repeat_interleave(heads // x.kv_heads, 1) for c in (x.k, x.v))   # [keys, heads, dim]
        key, place = torch.arange(len(pages), device="cuda"), torch.arange(n, device="cuda")
        j = key - start
        if mask is None:
            named = j <= place[:, None]
        else:
            words = mask.shape[1]
            named = (mask[lo:hi][:, (j // 64).clamp(0, words - 1)] >> (j % 64) & 1 == 1) & (j < 64 * words)
        see = ((j < 0) | named) & (pages >= 0)
        s = torch.einsum("nhd,khd->hnk", q[lo:hi].double(), k) * scale
        size = torch.nan_to_num(torch.einsum("nhd,khd->hnk", q[lo:hi].double().abs(), k.abs()) * scale)
        size = torch.where(see, size, 0.0).amax(-1, keepdim=True) if len(pages) else size.new_zeros(heads, n, 1)
        s = torch.where(see, s, -INF)
        p = torch.softmax(s, -1).nan_to_num(0.0) if not bool(see.any(1).all()) else torch.softmax(s, -1)
        # what is not seen must not touch the row, whatever it is
        plain = torch.isfinite(v)
        o = torch.einsum("hnk,khd->nhd", p, torch.where(plain, v, 0.0))
        a = torch.einsum("hnk,khd->nhd", p, torch.where(plain, v, 0.0).abs())
        for kk in (~plain).any(-1).any(-1).nonzero()[:, 0].tolist():
            for nn in see[:, kk].nonzero()[:, 0].tolist():
                o[nn] += torch.where(plain[kk], 0.0, v[kk] * p[:, nn, kk, None])
        d = 2 * (x.dim + 8) * 2.0**-23 * size + 2.0**-19 + len(pages) * 2.0**-23
        out[lo:hi] = o
        tol[lo:hi] = a * (h + d.permute(1, 0, 2)) + h * o.abs() + SMALLEST[x.dtype]
    return out, tol


def check_attend(x, heads, mask=None, scale=None, by=1.0, q=None):
    q = x.rows(heads, by) if q is None else q
    out = torch.full_like(q, 77.0)
    got = cache.tree_attention(q, x.k, x.v, *x.where(), mask=mask, scale=scale, out=out)
    assert got is out
    want, tol = attend_reference(x, q, mask, scale)
    lo_hi = [(int(x.offsets[i]), int(x.offsets[i + 1])) for i in range(x.offsets.numel() - 1)]
    behind = torch.ones(x.tokens, dtype=torch.bool, device="cuda")
    for lo, hi in lo_hi:
        behind[max(lo, 0) : max(hi, 0)] = False
    assert bool((got[behind] == 77.0).all())            # rows of no sequence stay as they were
    got, want, tol = got[~behind].double(), want[~behind], tol[~behind]
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    wild = ~torch.isfinite(want)
    assert torch.equal(got[wild].nan_to_num(5.0, 6.0, 7.0), want[wild].nan_to_num(5.0, 6.0, 7.0))
    off = (got - want).abs()
    assert bool((off <= tol)[~wild].all()), (off / tol)[~wild].max()
    again = cache.tree_attention(q, x.k, x.v, *x.where(), mask=mask, scale=scale)
    assert torch.equal(again[~behind].double().nan_to_num(5.0), got.nan_to_num(5.0))      # the same call, the same bits
    return out


def trees(x, nodes, seed=1, deep=False):
    g = torch.Generator().manual_seed(seed)
    parents = torch.empty(x.tokens, dtype=torch.int32)
    for i in range(x.offsets.numel() - 1):
        lo, hi = x.offsets[i : i + 2].tolist()
        for j in range(hi - lo):
            parents[lo + j] = j - 1 if deep else int(torch.randint(-1, j, (1,), generator=g)) if j else -1
    parents[int(x.offsets[-1]) :] = 5
    return parents.cuda()


# --- trees -------------------------------------------------------------------------------------------------------------------

def mask_reference(parents, offsets, starts, words):
    mask, positions = {}, {}
    for i in range(len(offsets) - 1):
        lo, bits, depth = offsets[i], [], []
        for j in range(offsets[i + 1] - lo):
            up = parents[lo + j]
            up = up if 0 <= up < j else -1
            bits.append((bits[up] if up >= 0 else 0) | 1 << j)
            depth.append(depth[up] + 1 if up >= 0 else 0)
            x = bits[-1]
            mask[lo + j] = [(x >> 64 * w & (1 << 64) - 1) - (x >> 64 * w + 63 & 1) * (1 << 64) for w in range(words)]
            positions[lo + j] = starts[i] + depth[-1]
    return mask, positions


@pytest.mark.parametrize("deep", [False, True])
@pytest.mark.parametrize("new,nodes", [([1], 1), ([0, 3, 1, 0, 2], 3), ([63, 64, 65, 1], 65), ([256, 255, 129], 256), ([300], 40), ([1025, 7], 1025),
                                       ([2050, 2048, 2049], 2050), ([4096], 4096), ([5] * 700, 64)],
                         ids=lambda x: str(x)[:24])
def test_tree_mask(new, nodes, deep):
    x = Batch([7 * i for i in range(len(new))], new, 1, 8, 16, BF16, behind=3, width=1)
    parents = trees(x, nodes, deep=deep)
    mask, positions = cache.tree_mask(parents, x.offsets, x.starts, nodes)
    want, where = mask_reference(parents.tolist(), x.offsets.tolist(), x.starts.tolist(), (nodes + 63) // 64)
    n = sum(new)
    assert mask[:n].tolist() == [want[i] for i in range(n)]
    assert positions[:n].tolist() == [where[i] for i in range(n)]
    assert torch.equal(cache.tree_mask(parents, x.offsets, None, nodes)[1][:n], positions[:n] - torch.repeat_interleave(
        x.starts, x.offsets[1:] - x.offsets[:-1]))


@pytest.mark.parametrize("skip", [0, 1])
@pytest.mark.parametrize("words", [1, 2, 3, 4, 5, 6, 64])
def test_tree_mask_of_any_number_of_words(words, skip):
    """More words than a tree needs, and fewer; rows that begin on 8 bytes and not on 16."""
    new = [63, 64, 65, 128, 129, 255, 256, 257, 0, 1]
    x = Batch([0] * len(new), new, 1, 8, 16, BF16, width=1)
    parents = trees(x, 257)
    n = sum(new)
    out = torch.full((skip + n * words + 1,), 9, dtype=torch.int64).cuda()
    assert b.lda_tree_mask(parents.data_ptr(), x.offsets.data_ptr(), len(new), n, None, words, out.data_ptr() + 8 * skip, None) == b.LDA_OK
    torch.cuda.synchronize()
    want, _ = mask_reference(parents.tolist(), x.offsets.tolist(), [0] * len(new), max(words, 5))
    assert out[skip:-1].view(n, words).tolist() == [want[i][:words] for i in range(n)]
    assert out[:skip].tolist() == [9] * skip and int(out[-1]) == 9


def test_tree_mask_of_strange_parents_and_offsets():
    parents = torch.tensor([0, 5, -7, 2, 2**31 - 1, -(2**31), 4, 1], dtype=torch.int32).cuda()
    offsets = torch.tensor([0, 7, 7, 8], dtype=torch.int64).cuda()
    mask, positions = cache.tree_mask(parents, offsets, None, 64)
    assert mask[:, 0].tolist() == [1, 2, 4, 12, 16, 32, 16 + 64, 1]
    assert positions.tolist() == [0, 0, 0, 1, 0, 0, 1, 0]
    # sequences whose offsets do not run upwards inside the tokens are left out
    out = torch.full((8, 1), 9, dtype=torch.int64).cuda()
    offsets = torch.tensor([0, 2, -1, 3, 9, 5, 8], dtype=torch.int64).cuda()
    assert b.lda_tree_mask(parents.data_ptr(), offsets.data_ptr(), 6, 8, None, 1, out.data_ptr(), None) == b.LDA_OK
    torch.cuda.synchronize()
    assert out[:, 0].tolist() == [1, 2, 9, 9, 9, 1, 2, 2 + 4]      # (the last one's parent is the one before)


# --- appending ---------------------------------------------------------------------------------------------------------------

def turned(x, positions, inv_freq, interleaved):
    """Rotation in 64 bits, and its tolerance before the last rounding."""
    x = x.double()
    if inv_freq is None:
        return x, torch.zeros_like(x)
    n = inv_freq.numel()
    angle = (positions.double()[:, None] * inv_freq.double())[:, None]
    a, c = (x[..., 0 : 2 * n : 2], x[..., 1 : 2 * n : 2]) if interleaved else (x[..., :n], x[..., n : 2 * n])
    out, tol = x.clone(), torch.zeros_like(x)
    size = (a.abs() + c.abs()) * 2.0**-20
    first, second = a * torch.cos(angle) - c * torch.sin(angle), a * torch.sin(angle) + c * torch.cos(angle)
    if interleaved:
        out[..., 0 : 2 * n : 2], out[..., 1 : 2 * n : 2] = first, second
        tol[..., 0 : 2 * n : 2] = tol[..., 1 : 2 * n : 2] = size
    else:
        out[..., :n], out[..., n : 2 * n] = first, second
        tol[..., :n] = tol[..., n : 2 * n] = size
    return out, tol


def near(got, want, tol, dtype):
    off = (got.double() - want).abs()
    return bool((off <= tol * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * want.abs() + SMALLEST[dtype]).all())


def check_append(x, heads, rot, interleaved=False, positions=None, in_place=False, split=True):
    total = heads + 2 * x.kv_heads
    if split:       # views of one projection's rows
        q, k, v = x.rows(total).split([heads, x.kv_heads, x.kv_heads], 1)
    else:
        q, k, v = x.rows(heads) if heads else None, x.rows(x.kv_heads), x.rows(x.kv_heads)
    q = q if heads else None
    inv_freq = (1e4 ** (-torch.arange(0, rot, 2).double() / rot)).float().cuda() if rot else None
    want_k, want_v = x.k.double(), x.v.double()
    slots = torch.zeros(x.tokens, dtype=torch.int64, device="cuda")
    seen = torch.zeros(x.tokens, dtype=torch.bool, device="cuda")
    for i in range(x.offsets.numel() - 1):
        lo, hi = x.offsets[i : i + 2].tolist()
        slots[lo:hi] = max(int(x.starts[i]), 0) + torch.arange(hi - lo, device="cuda")
        seen[lo:hi] = True
    pos = slots if positions is None else positions
    turned_k, tol_k = turned(k, pos, inv_freq, interleaved)
    tol = torch.zeros_like(want_k)
    for i in range(x.offsets.numel() - 1):
        lo, hi = x.offsets[i : i + 2].tolist()
        pages, places = x.slots(i)
        first = max(int(x.starts[i]), 0)
        pages, places = pages[first:], places[first:]
        ok = pages >= 0
        for want, got in ((want_k, turned_k), (tol, tol_k), (want_v, v.double())):
            want[pages[ok], places[ok]] = got[lo : lo + len(pages)][ok]
    want_q, tol_q = turned(q, pos, inv_freq, interleaved) if heads else (None, None)
    out = None
    if heads:
        out = q if in_place else torch.full((x.tokens, heads, x.dim), 77.0, dtype=x.dtype, device="cuda")
        want_q[~seen] = q[~seen].double() if in_place else 77.0
        tol_q[~seen] = 0.0
    versions = x.k._version, x.v._version
    got = cache.append_cache(k, v, x.k, x.v, *x.where(), positions=positions, inv_freq=inv_freq, interleaved=interleaved, q=q, q_out=out)
    assert x.k._version > versions[0] and x.v._version > versions[1]
    assert torch.equal(x.v.double(), want_v)
    assert near(x.k, want_k, tol, x.dtype)
    if heads:
        assert got is out and near(got, want_q, tol_q, x.dtype)
    else:
        assert got is None


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("dim,rot", [(8, 0), (8, 8), (8, 2), (16, 16), (64, 64), (80, 32), (80, 40), (96, 96), (128, 128), (128, 6), (256, 256), (248, 100)])
def test_append(dim, rot, interleaved, dtype):
    x = Batch([0, 5, 31, 100], [3, 0, 40, 1], 3, dim, 8, dtype, seed=dim + rot, behind=2)
    check_append(x, 6, rot, interleaved)


@pytest.mark.parametrize("page", [1, 7, 24, 64, 1000])
@pytest.mark.parametrize("by_head", [False, True])
def test_append_to_pages_of_any_size(page, by_head):
    x = Batch([17, 999, 0], [9, 33, 70], 2, 64, page, BF16, seed=page, by_head=by_head)
    check_append(x, 0, 64, split=False)
    check_append(x, 4, 32, in_place=True, split=False)
    check_append(x, 4, 64, True, in_place=True)


@pytest.mark.parametrize("sequences", [1, 2, 33, 255, 256, 257, 1000])
def test_append_of_few_and_of_many_sequences(sequences):
    x = Batch([i % 50 for i in range(sequences)], [(i * 7) % 4 for i in range(sequences)], 1, 32, 16, F16, seed=sequences)
    check_append(x, 2, 32)


def test_append_at_far_positions():
    """An angle of 10^6 and more, to the last place."""
    x = Batch([0, 40], [30, 30], 2, 128, 16, F16)
    positions = torch.tensor([0, 1, -1, 7, 10**6 + 1, 2**20 - 1, 2**24 + 1, -(2**24) - 1] * 7 + [3] * 4, dtype=torch.int32).cuda()
    check_append(x, 2, 128, positions=positions)


def test_append_where_the_table_has_no_pages():
    x = Batch([0, 20, 9, 0], [40, 20, 30, 5], 2, 64, 16, BF16, seed=4)
    x.table[0, 1], x.table[1, 2], x.table[2, 0] = -1, x.k.shape[0], 2**31 - 1
    x.table = x.table[:, :2].contiguous()          # and slots behind its end
    check_append(x, 4, 64)
    x.starts[:] = torch.tensor([2**31 - 1, 2**31 - 20, -3, 0])
    check_append(x, 4, 0)


def test_offsets_that_run_nowhere_write_nothing():
    x = Batch([0, 0, 0], [4, 4, 4], 1, 64, 16, BF16)
    k, v = x.k.clone(), x.v.clone()
    x.offsets = torch.tensor([-5, 20, 13, 30], dtype=torch.int64).cuda()
    rows_ = x.rows(1)
    out = torch.full((x.tokens, 1, 64), 3.0, dtype=BF16, device="cuda")
    cache.append_cache(rows_, rows_, x.k, x.v, *x.where(), q=rows_, q_out=out)
    assert torch.equal(x.k, k) and torch.equal(x.v, v) and bool((out == 3.0).all())
    assert torch.equal(cache.tree_attention(rows_, x.k, x.v, *x.where(), out=out), torch.full_like(out, 3.0))


# --- attention ---------------------------------------------------------------------------------------------------------------

SHAPES = [([0], [1], 1, 1, 8, 16), ([1], [1], 1, 1, 64, 16), ([63, 64, 65, 0], [1, 1, 1, 1], 2, 6, 64, 16), ([0, 0, 0], [1, 64, 65], 1, 2, 128, 16),
          ([100, 7, 0, 300], [3, 0, 17, 1], 2, 8, 128, 24), ([1000], [5], 5, 15, 80, 24), ([4097, 1], [1, 33], 1, 8, 96, 64),
          ([513, 0, 77], [13, 40, 2], 3, 3, 256, 8), ([30_000], [1], 2, 16, 128, 16), ([10_000, 3, 500], [8, 8, 8], 4, 16, 64, 32),
          ([200] * 40, [1] * 40, 2, 4, 248, 16), ([5000], [70], 2, 16, 128, 128), ([33, 900], [256, 3], 1, 7, 72, 7), ([77], [30], 1, 40, 16, 1)]


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("starts,new,kv_heads,heads,dim,page", SHAPES, ids=str)
def test_attention(starts, new, kv_heads, heads, dim, page, tree, dtype):
    x = Batch(starts, new, kv_heads, dim, page, dtype, seed=dim + page, by_head=page % 16 == 8, behind=2)
    mask = cache.tree_mask(trees(x, max(new)), x.offsets, x.starts, max(new))[0] if tree else None
    check_attend(x, heads, mask, by=2.0)


@pytest.mark.parametrize("sequences", [1, 2, 127, 128, 129, 400])
def test_attention_of_few_and_of_many_sequences(sequences):
    x = Batch([(i * 37) % 300 for i in range(sequences)], [(i * 5) % 4 for i in range(sequences)], 2, 64, 16, BF16, seed=sequences)
    check_attend(x, 8)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 4, 20, 64])
def test_any_mask(dim, new, dtype):
    """Masks that are no trees: rows that name nothing, everything, what lies behind them and places that are none."""
    x = Batch([0, 0, 70, 128, 1], [new] * 5, 2, dim, 16, dtype, seed=dim + new)
    g = torch.Generator().manual_seed(new)
    mask = torch.randint(-(2**63), 2**63 - 1, (x.tokens, 2), generator=g).cuda()
    mask[0], mask[new], mask[2 * new + new // 2] = 0, 0, 0
    mask[3 * new] = -1
    out = check_attend(x, 8, mask)
    assert bool((out[0] == 0).all()) and bool((out[new] == 0).all())      # no context, nothing named
    check_attend(x, 8, mask[:, :1])                                        # rows of a wider matrix
    check_attend(x, 2, torch.zeros_like(mask))


@pytest.mark.parametrize("dim,heads,new", [(64, 2, 5), (128, 4, 1), (128, 16, 40), (256, 2, 9)])
def test_what_is_not_seen_does_not_touch_a_row(dim, heads, new):
    x = Batch([0, 50, 64], [new] * 3, 2, dim, 16, F16, seed=3)
    mask = cache.tree_mask(trees(x, new), x.offsets, None, new)[0]
    # all slots that no sequence has
    used = torch.zeros(x.k.shape[:2], dtype=torch.bool, device="cuda")
    for i in range(3):
        pages, places = x.slots(i)
        used[pages, places] = True
    x.k[~used], x.v[~used] = NAN, NAN
    check_attend(x, heads, mask)
    # new tokens that some see and others do not
    for i, (kind, place) in enumerate(((NAN, new - 1), (INF, new // 2), (-INF, 0))):
        pages, places = x.slots(i)
        first = int(x.starts[i])
        x.v[pages[first + place], places[first + place], :, 1 + i] = kind
        x.k[pages[first + new - 1], places[first + new - 1], 0, 3] = NAN
    got = check_attend(x, heads, mask)
    if new > 1:
        assert bool(torch.isfinite(got[0]).all()) and bool(torch.isnan(got[new - 1]).any())


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
def test_scores_of_any_size(dtype):
    """Scores around 10^4, all alike, rows that one key has to itself, rows of 20 000 keys of next to no weight."""
    x = Batch([20_000, 100, 100], [2, 2, 2], 1, 64, 16, dtype, seed=9)
    check_attend(x, 2, scale=1.0, by=8.0)
    q = x.rows(2)
    q[:] = 0
    check_attend(x, 2, q=q)
    check_attend(x, 2, scale=1e-6)
    pages, places = x.slots(0)
    x.k[pages[777], places[777], 0] = 20.0
    q[:] = 20.0
    check_attend(x, 2, q=q, scale=0.002)


def test_a_key_at_infinity():
    x = Batch([40, 40], [1, 1], 1, 64, 16, F16)
    pages, places = x.slots(0)
    x.k[pages[3], places[3], 0, 5] = INF
    q = x.rows(1).abs()
    got = cache.tree_attention(q, x.k, x.v, *x.where())
    assert bool(torch.isnan(got[0]).all()) and bool(torch.isfinite(got[1]).all())


def test_keys_on_no_page_are_left_out():
    x = Batch([100, 300, 40, 5], [3, 3, 30, 2], 2, 64, 16, BF16, seed=8)
    x.table[0, 2], x.table[1, 0], x.table[1, 5], x.table[2, 4] = -1, x.k.shape[0], -(2**31), 2**31 - 1
    check_attend(x, 4)
    x.table[3] = -1
    out = check_attend(x, 4)
    assert bool((out[-2:] == 0).all())
    x.table = x.table[:, :4].contiguous()          # slots behind the table's end
    check_attend(x, 4)
    x.starts[1] = 2**31 - 2
    check_attend(x, 4)
    x.starts[2] = -9                                # counts as 0
    check_attend(x, 4)
    x.table = x.table[:, :0].contiguous()
    out = cache.tree_attention(x.rows(4), x.k, x.v, *x.where())
    assert bool((out == 0).all())


@pytest.mark.parametrize("kv_heads,heads", [(1, 1), (1, 64), (8, 8), (5, 35), (16, 128)])
def test_groups_of_any_size(kv_heads, heads):
    x = Batch([130, 64, 0], [1, 6, 2], kv_heads, 128, 16, BF16, seed=heads)
    check_attend(x, heads)


def test_strides():
    x = Batch([50, 3], [4, 7], 2, 64, 16, F16)
    wide = x.rows(12)
    check_attend(x, 4, q=wide[:, 3:7])
    q = torch.randn(4, x.tokens, 64, generator=x.g).to(F16).cuda().transpose(0, 1)
    check_attend(x, 4, q=q)
    check_attend(x, 4, q=x.rows(1).expand(-1, 4, -1))          # one head for all
    # a cache whose values lie otherwise than its keys, both inside of larger tensors
    big = torch.full((x.k.shape[0] + 2, 2, 3, 16, 72), NAN, dtype=F16, device="cuda")
    big[2:, 1, :2, :, 8:] = x.v.transpose(1, 2)
    x.v = big[2:, 1, :2, :, 8:].transpose(1, 2)
    check_attend(x, 4)
    check_append(x, 4, 64)
    one = Batch([5], [1], 1, 64, 16, F16, extra_pages=0)
    one.k, one.v = one.k.as_strided(one.k.shape, (3, 64, 5, 1)), one.v.as_strided(one.v.shape, (1, 64, 1, 1))     # strides that are never taken
    check_attend(one, 1)
    table = torch.full((2, 40), -1, dtype=torch.int32, device="cuda")
    table[:, 3 : 3 + x.table.shape[1]] = x.table
    x.table = table[:, 3 : 3 + x.table.shape[1]]
    check_attend(x, 2)


def test_a_cache_of_more_than_2_to_32_elements():
    pages, page, kv_heads, dim = 70_000, 64, 8, 128            # 4.6e9 elements, 9 GB each
    k, v = (torch.zeros(pages, page, kv_heads, dim, dtype=BF16, device="cuda") for _ in range(2))
    x = Batch([500, 90], [5, 1], kv_heads, dim, page, BF16)
    small_k, small_v, small_table = x.k, x.v, x.table.clone()
    far = pages - small_k.shape[0]
    k[far:], v[far:] = small_k, small_v
    x.table = torch.where(small_table >= 0, small_table + far, -1).to(torch.int32)
    x.k, x.v = k, v
    check_attend(x, 16)
    rows_ = x.rows(kv_heads)
    cache.append_cache(rows_, rows_, k, v, *x.where(), inv_freq=torch.ones(64, device="cuda"))
    cache.append_cache(rows_, rows_, small_k, small_v, small_table, x.starts, x.offsets, inv_freq=torch.ones(64, device="cuda"))
    assert torch.equal(k[far:], small_k) and torch.equal(v[far:], small_v)
    assert not bool(k[:4].any()) and not bool(v[far - 4 : far].any())


# --- streams and graphs ------------------------------------------------------------------------------------------------------

def test_nothing_to_do():
    x = Batch([3], [0], 2, 64, 16, F16)
    q = x.rows(4)
    assert cache.tree_attention(q, x.k, x.v, *x.where()).shape == (0, 4, 64)
    assert cache.append_cache(x.rows(2), x.rows(2), x.k, x.v, *x.where(), q=q).shape == (0, 4, 64)
    x = Batch([], [], 2, 64, 16, F16, behind=3, width=1)
    out = torch.full((3, 4, 64), 5.0, dtype=F16, device="cuda")
    assert bool((cache.tree_attention(x.rows(4), x.k, x.v, *x.where(), out=out) == 5.0).all())
    cache.append_cache(x.rows(2), x.rows(2), x.k, x.v, *x.where())
    mask, positions = cache.tree_mask(torch.zeros(0, dtype=torch.int32, device="cuda"), x.offsets, None, 5)
    assert mask.shape == (0, 1) and positions.shape == (0,)
    empty = torch.zeros(0, 16, 2, 64, dtype=F16, device="cuda")      # no pages at all
    x = Batch([3, 0], [2, 1], 2, 64, 16, F16)
    assert not bool(cache.tree_attention(x.rows(4), empty, empty, *x.where()).any())
    cache.append_cache(x.rows(2), x.rows(2), empty, empty, *x.where())


def step(x, q, k, v, inv_freq, parents, nodes):
    mask, positions = cache.tree_mask(parents, x.offsets, x.starts, nodes)
    q = cache.append_cache(k, v, x.k, x.v, *x.where(), positions=positions, inv_freq=inv_freq, q=q)
    return cache.tree_attention(q, x.k, x.v, *x.where(), mask=mask)


def test_two_streams_and_two_graphs_at_once():
    """Calls that overlap have workspaces of their own; a replayed graph sees what its tensors hold then."""
    batches = [Batch([3000, 10, 700], [9, 4, 1], 2, 128, 16, BF16, seed=s) for s in range(2)]
    inv_freq = (1e4 ** (-torch.arange(0, 128, 2).double() / 128)).float().cuda()
    ins = [(x.rows(8), x.rows(2), x.rows(2), inv_freq, trees(x, 9), 9) for x in batches]
    want = [step(x, *i) for x, i in zip(batches, ins)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = []
        for x, i, s in zip(batches, ins, streams):
            with torch.cuda.stream(s):
                got.append(step(x, *i))
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want))
    graphs, outs = [], []
    for x, i in zip(batches, ins):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(x, *i))
        graphs.append(g)
    for x, i in zip(batches, ins):
        i[0].copy_(x.rows(8))
        x.starts[0] -= 100
    want = [step(x, *i) for x, i in zip(batches, ins)]
    torch.cuda.synchronize()
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(outs, want))
