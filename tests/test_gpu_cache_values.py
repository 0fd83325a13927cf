"""Attention over a paged cache where values are infinite or no numbers: what a row does not see does not touch it, wherever it lies."""
import pytest
import torch

from test_gpu_cache import BF16, F16, INF, NAN, Batch, check_attend, trees
from paper_1412_1576_b200 import cache

pytestmark = pytest.mark.gpu

# (contexts, new tokens, heads of the cache, query heads, sequences without tokens behind them: rows of a tile go by the average).  So many heads
# that each of 148 runs of tiles has more than one item's, and a tile with such values has others behind it.
LONG = [([100, 70], [64, 64], 128, 512, 0),     # 256 rows, both teams have each tile of keys
        ([37, 5], [400, 130], 64, 64, 0),       # the same, and items of fewer rows among them
        ([37], [400], 64, 64, 15),              # 64 rows
        ([37], [600], 64, 64, 40)]              # 32 rows


def batch(starts, new, kv_heads, empty, dim, dtype, page=16):
    return Batch(starts + [0] * empty, new + [0] * empty, kv_heads, dim, page, dtype, seed=dim + empty)


def put(x, i, slot, column, value):
    pages, places = x.slots(i)
    x.v[pages[slot], places[slot], :, column] = value


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("starts,new,kv_heads,heads,empty", LONG, ids=str)
def test_values_in_any_of_several_tiles_of_new_tokens(starts, new, kv_heads, heads, empty, dim, tree, dtype):
    """One kind in the first of the tiles, which rows behind it see, then all kinds in the first, a middle and the last one, some of them alone in
    their column and some together."""
    x = batch(starts, new, kv_heads, empty, dim, dtype)
    mask = cache.tree_mask(trees(x, max(new)), x.offsets, None, max(new))[0] if tree else None
    q = x.rows(heads, by=0.5)
    put(x, 0, starts[0] + 3, 5, NAN)
    check_attend(x, heads, mask, q=q)
    for i, n in enumerate(new):
        for j, (place, kind) in enumerate([(2, INF), (7, -INF), (n // 2, -INF), (n // 2 + 1, NAN), (n - 2, INF), (n - 1, NAN)]):
            put(x, i, starts[i] + place, 8 + j, kind)
            put(x, i, starts[i] + place, 40 + j % 3, kind)
    got = check_attend(x, heads, mask, q=q)
    # (of a chain, the first tokens see none of it)
    assert tree or bool(torch.isfinite(got[:2]).all()) and bool(torch.isinf(got[3:7]).any())


@pytest.mark.parametrize("empty,new", [(0, 40), (12, 300), (29, 300)])
@pytest.mark.parametrize("dim", [64, 128])
def test_values_beside_a_missing_page(empty, new, dim):
    """A tile in the middle of a context, of which a page is missing."""
    x = batch([1000], [new], 64, empty, dim, BF16)
    x.table[0, 17] = -1                     # slots 272 .. 287
    put(x, 0, 260, 3, INF)
    put(x, 0, 300, 4, -INF)
    put(x, 0, 383, 5, NAN)
    heads = 64 if empty else 512
    got = check_attend(x, heads, q=x.rows(heads, by=0.5))
    assert bool((got[:, :, 3] == INF).all()) and bool((got[:, :, 4] == -INF).all()) and bool(torch.isnan(got[:, :, 5]).all())


# (the same operator by other rows of a tile, and by the kernel for other pages and heads; one head of the cache, whose keys several CTAs share, and many)
@pytest.mark.parametrize("new,empty,group,dim,page", [(40, 0, 8, 64, 16), (40, 0, 8, 128, 16), (40, 0, 2, 128, 16), (24, 0, 1, 128, 16), (24, 1, 2, 64, 16),
                                                      (1, 0, 1, 64, 16), (1, 0, 8, 128, 16), (5, 0, 3, 80, 24), (1, 0, 8, 128, 4), (5, 0, 4, 256, 16), (40, 0, 8, 64, 4)])
@pytest.mark.parametrize("kv_heads", [1, 48])
@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
def test_infinities_in_a_context_that_all_see(new, empty, group, dim, page, kv_heads, dtype):
    """In the context's tiles nothing is hidden; an infinity among the values is the row's output in its column, and not a NaN."""
    x = batch([1500], [new], kv_heads, empty, dim, dtype, page)
    heads = group * kv_heads
    for slot, column, kind in [(0, 1, INF), (130, 2, -INF), (700, 3, INF), (1400, 3, INF), (64, 4, INF), (1000, 4, -INF), (900, 5, NAN), (901, 5, INF),
                               (1407, 6, INF), (1408, 7, -INF), (1499, 7, -INF)]:
        put(x, 0, slot, column, kind)
    got = check_attend(x, heads, q=x.rows(heads, by=0.5))
    assert bool((got[:, :, 1] == INF).all()) and bool((got[:, :, 2] == -INF).all()) and bool(torch.isnan(got[:, :, 4:6]).all())
    put(x, 0, 1500, 9, -INF)               # with one among the new tokens, and a row of which nothing is a number
    q = x.rows(heads, by=0.5)
    q[0, 0, 0] = NAN
    got = check_attend(x, heads, q=q)
    assert bool(torch.isnan(got[0, 0]).all())


def test_an_infinity_at_the_end_of_the_longest_sequence():
    """Numbers of keys up to 2^31 - 9: all entries of the table name one page, and a last one another, with the infinity."""
    width = 2**28 - 1
    k = torch.zeros(2, 8, 1, 8, dtype=F16, device="cuda")
    v = torch.ones_like(k)
    v[1, 3, 0, 2], v[1, 5, 0, 4] = INF, -INF
    table = torch.zeros(1, width, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    starts = torch.tensor([8 * width - 1], dtype=torch.int32).cuda()
    got = cache.tree_attention(torch.ones(1, 4, 8, dtype=F16, device="cuda"), k, v, table, starts, torch.tensor([0, 1]).cuda())
    want = torch.ones(8)
    want[2], want[4] = INF, -INF
    # (the norm's and the outputs' sums are of single precision, 2^31 / 148 terms each: the same terms in other orders)
    assert torch.equal(torch.isinf(got[0].cpu()), torch.isinf(want).expand(4, 8)) and bool((got[0, :, 2] == INF).all()) and bool((got[0, :, 4] == -INF).all())
    assert not bool(torch.isnan(got).any())


@pytest.mark.parametrize("new,empty,heads,dim,page", [(300, 0, 64, 64, 16), (300, 15, 32, 128, 16), (300, 40, 32, 64, 16), (300, 0, 8, 64, 4), (40, 0, 8, 256, 16)])
def test_an_infinity_of_next_to_no_weight(new, empty, heads, dim, page):
    """Among the new tokens' values, at keys whose weights are far below what single precision has: those who see it have it, the others do not."""
    x = batch([200], [new], heads, empty, dim, BF16, page)
    q = x.rows(heads)
    q[:] = 2.0
    pages, places = x.slots(0)
    x.k[:] = 1.0
    x.k[pages[200 + 5], places[200 + 5]] = -6.0       # (scores lower by 14 times the head's values)
    x.v[pages[200 + 5], places[200 + 5], :, 3] = INF
    got = cache.tree_attention(q, x.k, x.v, *x.where(), scale=1.0)[:new]
    assert bool((got[5:, :, 3] == INF).all()) and bool(torch.isfinite(got[:5]).all()) and bool(torch.isfinite(got[:, :, :3]).all())
