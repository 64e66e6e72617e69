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


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_what_a_row_attends_shows_where_it_is(ema, out_dtype):
    """NaN in a key makes its pair's outputs NaN, NaN or an infinity in a value its channel."""
    inf, nan = 0x7F80, 0x7FC0
    c = SmallCache(ema, [70, 40], 4, 16, "bf16", seed=55)
    try:
        c.poke(1, 0, 33, 0, 5, inf)
        c.poke(1, 0, 34, 1, 6, nan)
        c.poke(0, 1, 3, 3, 0, nan)
        c.upload()
        lam = torch.full((4,), 0.5, device="cuda")
        out = torch.zeros((2, 4, 2 * D), dtype=out_dtype, device="cuda")
        ema.paged_diff_attention(c.h, dev16(c.queries(2, 8), "bf16"), c.table_dev, c.lens_dev, lam,
                                 out)
        finite = torch.isfinite(out).cpu().numpy()
        want = np.ones((2, 4, 2 * D), bool)
        want[0, :2, [5, D + 6]] = False                  # heads 0 and 1 read KV heads 0 and 1
        want[1, 2:] = False                              # heads 2 and 3 KV heads 2 and 3
        assert np.array_equal(finite, want)
        assert torch.isnan(out[1, 2:]).all() and torch.isnan(out[0, :2, D + 6]).all()
    finally:
        c.close()
