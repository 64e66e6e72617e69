"""Starts at the ends of their type: rows of attention calls are clamped to what is there."""
import numpy as np
import pytest
import torch

from ops_harness import D, SmallCache, dev16, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("maps", [1, 2])
@pytest.mark.parametrize("B", [3, 600])
def test_the_lowest_and_highest_starts(maps, B):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema
    c = SmallCache(ema, [40] * B, 2, 16, "bf16", seed=1)
    try:
        q, lam = dev16(c.queries(9, 4), "bf16"), torch.ones(2, device="cuda")
        starts = np.zeros(B + 1, np.int64)
        starts[1:4] = 2 ** 31 - 1, -2 ** 31, 9           # past the rows, descends, negative
        starts[4:] = 9
        o = torch.full((9, 4 // maps, maps * D), 7.0, device="cuda")
        args = (c.h, q, i32(starts), c.table_dev, c.lens_dev)
        if maps == 1:
            ema.paged_prompt_attention(*args, o)
        else:
            ema.paged_diff_prompt_attention(*args, lam, o)
        assert ema.slice_device_errors(c.h) == 3
        assert torch.isfinite(o).all()
    finally:
        c.close()
