"""Single-token differential attention where one map's key holds an infinity whose score is
-inf: that token has no weight in that map, and the other map does not see it."""
import numpy as np
import pytest
import torch

from ops_harness import D, SmallCache, dev16
from oracle import ops as oops
from ops_harness import assert_close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


@pytest.mark.parametrize("heads", [1, 3, 8, 16])
@pytest.mark.parametrize("kv_head", [0, 1])
def test_an_infinite_key_stays_in_its_map(ema, heads, kv_head):
    c = SmallCache(ema, [70], 2, 16, "bf16", seed=54)
    try:
        q16 = c.queries(1, 2 * heads)
        q16[:, :, 7] = 0x3F80                            # 1.0
        c.poke(0, 0, 33, kv_head, 7, 0xFF80)             # -inf
        c.upload()
        lam = np.linspace(0.2, 0.8, heads).astype(np.float32)
        out = torch.zeros((1, heads, 2 * D), device="cuda")
        ema.paged_diff_attention(c.h, dev16(q16, "bf16"), c.table_dev, c.lens_dev,
                                 torch.tensor(lam, device="cuda"), out)
        with np.errstate(all="ignore"):
            ref, mass = oops.prompt_attention(q16, [0, 1], c.table, c.lens, c.read_block, 2, D, 16,
                                              "bf16", lam=lam)
        assert np.isfinite(ref).all()
        assert_close(out, ref, mass, torch.float32, "bf16", 70)
    finally:
        c.close()
