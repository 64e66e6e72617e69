"""Lengths at the ends of their type: the tokens before a tree of more nodes than its request
has tokens are a negative number, however short the request is said to be."""
import numpy as np
import pytest
import torch

from ops_harness import D, i32

pytestmark = pytest.mark.gpu


def test_base_of_the_lowest_lengths():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema
    low, high = -2 ** 31, 2 ** 31 - 1
    sizes, lens = [3, 3, 1, 3, 64], [low, low + 2, low + 1, low + 3, high]
    starts = np.concatenate([[0], np.cumsum(sizes)])
    h = ema.slice_create(1, D, 16, "bf16", 0, 4 * 8192, 0)
    try:
        parents = np.concatenate([np.arange(n) - 1 for n in sizes])
        mask = torch.zeros((74, 1), dtype=torch.int64, device="cuda")
        pos, base = i32(np.zeros(74)), i32(np.zeros(5))
        ema.tree_tables(h, i32(parents), i32(starts), i32(lens), mask, pos, base)
        want = [max(n, low + k) - k for n, k in zip(lens, sizes)]
        assert base.cpu().tolist() == want == [low, low, low, low, high - 64]
        assert pos.cpu().tolist() == [x + i for x, n in zip(want, sizes) for i in range(n)]
        assert ema.slice_device_errors(h) == 4
    finally:
        ema.slice_destroy(h)
