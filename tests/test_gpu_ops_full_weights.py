"""16-bit outputs of softmax weights kept to 32-bit accuracy: the 32-bit output's values, each
rounded once."""
import numpy as np
import pytest
import torch

from ops_harness import D, SmallCache, dev16, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


@pytest.mark.parametrize("lens,new", [([40, 129], [40, 100]), ([3000], [9])])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("op", ["prompt", "diff", "diff-prompt"])
def test_full_weights_round_the_32_bit_output(ema, op, dtype, lens, new):
    c = SmallCache(ema, lens, 2, 16, dtype, seed=60)
    try:
        rows = len(lens) if op == "diff" else sum(new)
        maps = 1 if op == "prompt" else 2
        q, starts = dev16(c.queries(rows, 8), dtype), i32(np.concatenate([[0], np.cumsum(new)]))
        lam, norm = torch.linspace(0.1, 0.9, 4, device="cuda"), torch.ones(2 * D, device="cuda")

        def call(out_dtype, **kw):
            out = torch.zeros((rows, 8 // maps, maps * D), dtype=out_dtype, device="cuda")
            if op == "prompt":
                ema.paged_prompt_attention(c.h, q, starts, c.table_dev, c.lens_dev, out, **kw)
            elif op == "diff":
                ema.paged_diff_attention(c.h, q, c.table_dev, c.lens_dev, lam, out, norm_eps=1e-5,
                                         norm_weight=norm, **kw)
            else:
                ema.paged_diff_prompt_attention(c.h, q, starts, c.table_dev, c.lens_dev, lam, out,
                                                norm_weight=norm, norm_eps=1e-5, **kw)
            return out

        full = call(torch.float32)
        assert torch.equal(full, call(torch.float32, full_weights=True))
        for t in (torch.bfloat16, torch.float16):
            assert torch.equal(full.to(t), call(t, full_weights=True))
        once = call(full.dtype if op == "diff" else torch.bfloat16)
        assert op == "diff" or not torch.equal(full.to(torch.bfloat16), once)
    finally:
        c.close()
