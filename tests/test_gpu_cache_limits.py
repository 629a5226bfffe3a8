"""Attention over the paged cache where it can go wrong by its schedule or its number range (GPU).

Tolerances are those of tests/test_gpu_cache_attn.py.
"""

import pytest

from tests.gpu_util import announce
from tests.test_gpu_cache_attn import call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d,page", [(136, 16), (160, 7), (256, 16), (256, 100)])
def test_waves_of_a_tile_that_leave_steps_out(d, page, dtype):
    """Heads above 128, tiles of many rows: with a window the tile's first steps are seen by its first wave alone, so the
    others pass them without products and are the first to store the next keys.  Every call gives the same bits, those
    of the formula."""
    import torch

    announce(f"cache attn: waves apart, d={d} pages of {page} {dtype}")
    c = make([(129, 700), (260, 300), (70, 70)], dtype=dtype, hq=4, hkv=2, d=d, page=page, seed=11)
    for window in (0, 1, 40, 90):
        o, s = call(c, window=window)
        check(c, o, s, window=window)
        for _ in range(10):
            o2, s2 = call(c, window=window)
            assert torch.equal(o, o2) and torch.equal(s, s2)
