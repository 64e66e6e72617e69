"""Tables far wider than the lengths, as a cache's are: the width decides how the work is
cut, so parts without a token and more parts than tiles occur."""
import numpy as np
import pytest
import torch

from ops_harness import SmallCache
from test_gpu_ops import check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("lens,new,bs", [([1], [1], 16), ([70, 0, 200], [33, 0, 1], 16),
                                         ([700, 65] * 3, [90, 65] * 3, 32), ([5, 300], [5, 2], 128)])
@pytest.mark.parametrize("maps,single", [(1, False), (2, False), (2, True)])
@pytest.mark.parametrize("extra", [400, 2500])
def test_wide_tables(ema, lens, new, bs, maps, single, out, extra):
    c = SmallCache(ema, lens, 2, bs, "bf16", seed=55, extra_width=extra)
    try:
        new = [1] * len(lens) if single else new
        check_attention(ema, c, new, 8, out, maps, norm=maps == 2, single=single, pad=0 if single else 2)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()


def test_the_width_changes_how_the_work_is_cut(ema):
    c = SmallCache(ema, [70], 2, 16, "bf16", seed=56)
    try:
        sizes = [ema.paged_prompt_workspace(c.h, 33, 1, 8, w) for w in (5, 405, 2505)]
        assert sizes[0] == 0 and sizes[2] > sizes[1] > 0
    finally:
        c.close()
