"""Appending to a paged cache: offsets that do not run upwards leave out the sequences whose own they are, and no others."""
import pytest
import torch

from test_gpu_cache import BF16, Batch
from paper_1412_1576_b200 import cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offsets", [[0, 2, -1, 3, 9, 5, 8], [2, 5, 0, 2], [0, 100, 4, 8], [4, 8, 0, 4, 3], [8, 0, 0, 8, 8], [-1, 4, 8], [0, 3, 2**40, 3, 8],
                                     [-(2**62), 0, 2**62, 8, 5, 8], [9, 0] + [300] * 300 + [0, 5, 5, 1, 300, 5, 8]], ids=lambda x: str(x)[:24])
def test_only_the_sequences_of_bad_offsets_are_left_out(offsets):
    tokens, n = 8, len(offsets) - 1
    x = Batch([3 * (i % 9) for i in range(n)], [8] * n, 2, 64, 16, BF16, seed=n)
    x.tokens = tokens
    q, k, v = (x.rows(h) for h in (4, 2, 2))
    inv_freq = (1e4 ** (-torch.arange(0, 64, 2).double() / 64)).float().cuda()
    want_k, want_v, want_q = x.k.clone(), x.v.clone(), torch.full_like(q, 77.0)
    valid = [i for i in range(n) if 0 <= offsets[i] <= offsets[i + 1] <= tokens]
    assert sum(offsets[i + 1] - offsets[i] for i in valid) <= tokens      # no token is claimed twice
    for i in valid:        # by itself
        one = torch.tensor(offsets[i : i + 2]).cuda()
        cache.append_cache(k, v, want_k, want_v, x.table[i : i + 1], x.starts[i : i + 1], one, inv_freq=inv_freq, q=q, q_out=want_q)
    got_q = torch.full_like(q, 77.0)
    cache.append_cache(k, v, x.k, x.v, x.table, x.starts, torch.tensor(offsets).cuda(), inv_freq=inv_freq, q=q, q_out=got_q)
    assert torch.equal(x.k, want_k) and torch.equal(x.v, want_v) and torch.equal(got_q, want_q)
    assert bool((got_q == 77.0).any()) == (sum(offsets[i + 1] - offsets[i] for i in valid) < tokens)


def test_many_sequences_and_tokens():
    """Several rounds of sequences, empty ones among them, and more than one CTA's tokens."""
    lengths = [(i * 7) % 4 for i in range(1500)]
    x = Batch([i % 40 for i in range(1500)], lengths, 1, 8, 16, BF16, seed=1)
    rows = x.rows(1)
    cache.append_cache(rows, rows, x.k, x.v, x.table, x.starts, x.offsets)
    seq = torch.repeat_interleave(torch.arange(1500).cuda(), torch.tensor(lengths).cuda())
    slot = x.starts[seq].long() + torch.arange(x.tokens).cuda() - x.offsets[seq]
    pages = x.table[seq, slot // 16].long()
    assert torch.equal(x.k[pages, slot % 16], rows) and torch.equal(x.v[pages, slot % 16], rows)
