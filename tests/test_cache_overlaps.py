"""Operators on a paged cache: what is written must not share its places, and where that is refused (before anything reaches a GPU)."""
import pytest

from paper_1412_1576_b200 import binding as b
from test_cache_refusals import P, append, attend

# rows of outputs at address `out` with strides `os`, of 3 tokens with 4 heads of 64 values; queries at P with strides (256, 64)
OVERLAPS = [dict(os=(0, 64)), dict(os=(256, 0)), dict(os=(0, 0)), dict(os=(256, 56)), dict(os=(248, 64)), dict(os=(64, 64)), dict(os=(64, 128)),
            dict(out=P + 16), dict(out=P + 128), dict(out=P - 16), dict(out=P + 512), dict(out=P + 3 * 512 - 16), dict(out=P - 3 * 512 + 16),
            dict(out=P, os=(64, 192)), dict(out=P + 512, os=(512, 64)), dict(out=P - 512, os=(512, 64)),
            dict(qs=(1024, 64), os=(1024, 64), out=P + 16), dict(qs=(1024, 64), os=(1024, 64), out=P + 2 * 1024 + 496),
            dict(qs=(1024, 64), os=(1024, 64), out=P + 2 * (1024 - 192)), dict(qs=(1024, 64), os=(1024, 64), out=P - 2 * (1024 + 64)),
            dict(qs=(0, 0), os=(256, 64), out=P), dict(qs=(0, 64), os=(256, 64), out=P - 512)]


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("bad", OVERLAPS, ids=str)
def test_rows_of_outputs_that_overlap_are_refused(call, bad):
    assert call(**dict(dict(out=P + (1 << 20)), **bad)) == b.LDA_EINVAL


@pytest.mark.parametrize("steps", [(0, 128, 64), (2048, 0, 64), (2048, 128, 0), (2040, 128, 64), (2048, 120, 64), (2048, 128, 56), (64, 64, 64), (2048, 64, 1016),
                                   (64, 320, 320), (128, 128, 64)], ids=str)
def test_a_cache_that_overlaps_itself_is_not_written_to(steps):
    assert append(key_steps=steps) == append(value_steps=steps) == b.LDA_EINVAL
