"""Attention over a paged cache: a wait inside the kernel that gives up is seen by the caller."""
import pytest
import torch

from test_gpu_cache import BF16, F16, Batch, check_attend
from paper_1412_1576_b200 import binding as b
from paper_1412_1576_b200 import build, cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def impatient(tmp_path_factory):
    """The library built so that every wait of the kernel gives up at once: nothing is copied and no product issued."""
    return b.load_library(build.build_library(extra_flags=("-DLDA_WAIT_POLLS=0",), out=str(tmp_path_factory.mktemp("lib") / "liblda_impatient.so")))


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("starts,new,kv_heads,heads", [([2000, 3, 0], [1, 1, 1], 2, 8), ([700], [8], 2, 6), ([300, 4], [64, 33], 2, 8), ([40], [400], 1, 1),
                                                       ([30_000], [2], 1, 4), ([100] * 60, [30] * 60, 8, 8)], ids=lambda x: str(x)[:24])
def test_rows_whose_waits_gave_up_are_nan(impatient, monkeypatch, starts, new, kv_heads, heads, dim, dtype):
    """In items that one CTA has and in those that several have and a join puts together; other rows stay, and the next call is right."""
    x = Batch(starts, new, kv_heads, dim, 16, dtype, behind=2)
    q = x.rows(heads)
    out = torch.full_like(q, 77.0)
    with monkeypatch.context() as m:
        m.setattr(b, "_lib", impatient)
        cache.tree_attention(q, x.k, x.v, *x.where(), out=out)
        torch.cuda.synchronize()
    n = sum(new)
    assert bool(torch.isnan(out[:n]).all()) and bool((out[n:] == 77.0).all())
    check_attend(x, heads, q=q)
