"""Relative 2-norm errors of attention over long float16 caches, where many small
weights make up a row.

What they may be. A score is 128 products of exact 16-bit values added up in 32 bits, in 8 steps of
the matrix cores that are each off by at most 2^-24 of the sum so far. With queries of
deviation 1/4 a sum has deviation 1/4 * sqrt(128) = 2.8 and stays below 16, so a score is off by
8 * 16 * 2^-24 = 7.6e-6, scaled by 1 / sqrt(128) 7e-7. The exponent's argument, below 32 in the
log2 domain, is rounded to 2^-24 * 32 = 2e-6, times ln 2 1.3e-6, and so is the maximum taken
from it; the exponential is off by 2^-23. 5e-6 a weight covers all of them. Two 16-bit parts
keep a weight to 2^-22 of it. Errors of different tokens multiply independent values, so a row's
norm is off by no more than its weights are, and twice as much where two maps are subtracted,
the second with a factor of 1/2: 1e-5.
A 16-bit output is off by half a step, 2^-11, and so is each of its weights."""
import numpy as np
import pytest
import torch

import synth
from ops_harness import D, SmallCache, dev16, i32
from oracle import ops as oops

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


def error(ema, op, n, rows, out_dtype, sink=0.0):
    """The worst relative 2-norm of a row. `sink`: how far the first token's score lies
    above the others', its value zero."""
    maps = 1 if op == "prompt" else 2
    c = SmallCache(ema, [n], 2, 256, "f16", seed=n)
    try:
        q16 = synth.round_to_16bit(0.25 * c.rng.standard_normal((rows, 4, D), dtype=np.float32),
                                   "f16")
        if sink:
            q16[..., 0] = synth.round_to_16bit(np.array([8.0], np.float32), "f16")[0]
            e = c.local.view(np.uint16).reshape(c.n_local, -1)
            for h in range(2):
                for t in range(n):
                    u, at = c.element(0, 0, t, h)
                    e[u, at[0]] = 0
                u, at = c.element(0, 0, 0, h)
                e[u, at] = 0
                e[u, at[0]] = synth.round_to_16bit(
                    np.array([sink * np.sqrt(128) / 8], np.float32), "f16")[0]
                u, at = c.element(1, 0, 0, h)
                e[u, at] = 0
            c.upload()
        lam = np.array([0.5, 0.5], np.float32)
        out = torch.empty((rows, 4 // maps, maps * D), dtype=out_dtype, device="cuda")
        q, starts, lam_dev = dev16(q16, "f16"), i32([0, rows]), torch.tensor(lam, device="cuda")
        if op == "prompt":
            ema.paged_prompt_attention(c.h, q, starts, c.table_dev, c.lens_dev, out)
        elif op == "diff":
            ema.paged_diff_attention(c.h, q, c.table_dev, c.lens_dev, lam_dev, out)
        else:
            ema.paged_diff_prompt_attention(c.h, q, starts, c.table_dev, c.lens_dev, lam_dev, out)
        ref, _ = oops.prompt_attention(q16, [0, rows], c.table, c.lens, c.read_block, 2, D, 256,
                                       "f16", lam=lam if maps == 2 else None)
        x = out.double().cpu().numpy()
        return float((np.linalg.norm(x - ref, axis=-1) / np.linalg.norm(ref, axis=-1)).max())
    finally:
        c.close()


@pytest.mark.parametrize("n,rows", [(2048, 5), (8191, 5), (60000, 2)])
def test_differential_chunks_of_many_small_weights(ema, n, rows):
    assert error(ema, "diff-prompt", n, rows, torch.float32) <= 1e-5
    assert error(ema, "diff-prompt", n, rows, torch.float16) <= 2 * 2.0 ** -11


# A first token that takes most of the weight and adds nothing, its score 12 above the others: they
# are off by 2^-25 of a scale in which the largest weight is 2^11 at least, 2.4e-6 of
# them; its own score of 12 * sqrt(128) before scaling by 8 * 136 * 2^-24 / sqrt(128) = 6e-6,
# which all of them share. With 5e-6 as above 1.3e-5, and twice that for two maps.
SINK, SINK_ERR = 12.0, 3e-5


@pytest.mark.parametrize("n,rows", [(2048, 5), (8191, 5), (60000, 2)])
def test_prompts_whose_first_token_takes_the_weight(ema, n, rows):
    assert error(ema, "prompt", n, rows, torch.float32, SINK) <= SINK_ERR


@pytest.mark.parametrize("n", [2048, 8191, 60000])
def test_single_tokens_whose_first_token_takes_the_weight(ema, n):
    assert error(ema, "diff", n, 1, torch.float32, SINK) <= SINK_ERR


@pytest.mark.parametrize("n,rows", [(2048, 5), (8191, 5), (60000, 2)])
def test_differential_chunks_whose_first_token_takes_the_weight(ema, n, rows):
    assert error(ema, "diff-prompt", n, rows, torch.float32, SINK) <= SINK_ERR
