"""Operators on a paged cache: outputs in their queries' places, beside them in the same rows, and in permuted tensors."""
import pytest
import torch

from test_gpu_cache import BF16, Batch
from paper_1412_1576_b200 import cache

pytestmark = pytest.mark.gpu


def places(x, heads):
    """Pairs of queries (to be filled) and outputs that share no place, or all of them."""
    n, d = x.tokens, x.dim
    rows = torch.zeros(n, 2 * heads, d, dtype=BF16, device="cuda")
    yield rows[:, :heads], rows[:, heads:]                              # two parts of the same rows
    yield rows[:, heads:], rows[:, :heads]
    yield rows[:, ::2], rows[:, 1::2]
    two = torch.zeros(2, heads, n, d, dtype=BF16, device="cuda").transpose(1, 2)
    yield two[0], two[1]                                                # head by head
    half = torch.zeros(2 * n, heads, d, dtype=BF16, device="cuda")
    yield half[::2], half[1::2]
    yield torch.zeros(n, heads, d, dtype=BF16, device="cuda"), two[0]
    yield rows[:, :heads], rows[:, :heads]
    yield two[1], two[1]


@pytest.mark.parametrize("starts,new,kv_heads,heads,page", [([500, 3], [9, 1], 2, 8, 16), ([3000], [70], 2, 8, 16), ([700, 90, 5], [1, 1, 1], 4, 4, 16),
                                                            ([300, 7], [20, 2], 2, 4, 4), ([1], [1], 1, 1, 16)])
def test_outputs_beside_and_in_their_queries_places(starts, new, kv_heads, heads, page):
    x = Batch(starts, new, kv_heads, 64, page, BF16)
    inv_freq = (1e4 ** (-torch.arange(0, 64, 2).double() / 64)).float().cuda()
    given, k, v = x.rows(heads), x.rows(kv_heads), x.rows(kv_heads)
    turned = cache.append_cache(k, v, x.k, x.v, *x.where(), inv_freq=inv_freq, q=given)
    want = cache.tree_attention(given, x.k, x.v, *x.where())
    for q, out in places(x, heads):
        same = q.data_ptr() == out.data_ptr()
        q.copy_(given)
        assert torch.equal(cache.append_cache(k, v, x.k, x.v, *x.where(), inv_freq=inv_freq, q=q, q_out=out), turned) and (same or torch.equal(q, given))
        q.copy_(given)
        assert torch.equal(cache.tree_attention(q, x.k, x.v, *x.where(), out=out), want) and (same or torch.equal(q, given))


def test_expanded_tensors_are_not_written_to():
    x = Batch([5, 9], [2, 3], 2, 64, 16, BF16)
    q, k = x.rows(4), x.rows(2)
    for out in (x.rows(1).expand(-1, 4, -1), q[:1].expand(5, -1, -1)):
        with pytest.raises(Exception, match="lda_append_cache"):
            cache.append_cache(k, k, x.k, x.v, *x.where(), q=q, q_out=out)
        with pytest.raises(Exception, match="lda_tree_attention"):
            cache.tree_attention(q, x.k, x.v, *x.where(), out=out)
    one = x.k[:1].expand_as(x.k)
    with pytest.raises(Exception, match="lda_append_cache"):
        cache.append_cache(k, k, one, x.v, *x.where())
    assert cache.tree_attention(q, one, x.v, *x.where()).shape == q.shape        # (reading is another matter)
