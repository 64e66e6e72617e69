"""What the kernels of prompts and differential attention do about arrays that are out of
range: block ids of no local block are left out, wherever they stand, and counted
once."""
import numpy as np
import pytest
import torch

import oracle
from ops_harness import D, SmallCache, dev16, i32
from oracle import ops as oops
from oracle.attention import _gather_sequence

pytestmark = pytest.mark.gpu
LAM = np.array([0.5, 0.25], np.float32)
OUT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


def attend(ema, c, op, q16, starts, table, out_dtype):
    rows = q16.shape[0]
    maps = 1 if op == "prompt" else 2
    out = torch.zeros((rows, 4 // maps, maps * D), dtype=out_dtype, device="cuda")
    q, table, lam = dev16(q16, c.dtype), i32(table), torch.tensor(LAM, device="cuda")
    if op == "prompt":
        ema.paged_prompt_attention(c.h, q, i32(starts), table, c.lens_dev, out)
    elif op == "diff":
        ema.paged_diff_attention(c.h, q, table, c.lens_dev, lam, out)
    else:
        ema.paged_diff_prompt_attention(c.h, q, i32(starts), table, c.lens_dev, lam, out)
    return out


def left_out(c, op, q16, row, b, seen, gone):
    """Row `row` of request b, which sees `seen` tokens but for those in the blocks `gone`."""
    K, V = _gather_sequence(c.read_block, c.table[b], int(c.lens[b]), 2, D, c.bs)
    keep = [t for t in range(seen) if t // c.bs not in gone]
    K, V = (oracle.to_float64(x, c.dtype)[:, keep] for x in (K, V))
    q = oracle.to_float64(q16[row], c.dtype)
    if op == "prompt":
        return np.stack([oops._weights(q[h], K[h // 2], D ** -0.5) @ V[h // 2] for h in range(4)])
    w = [oops._weights(q[h], K[h % 2], D ** -0.5) for h in range(4)]
    v = np.concatenate([V[0], V[1]], axis=1)
    return np.stack([(w[2 * h] - LAM[h] * w[2 * h + 1]) @ v for h in range(2)])


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("op", ["prompt", "diff", "diff-prompt"])
def test_a_bad_entry_far_into_the_table(ema, op, out):
    """Past the first 64 entries, with block 0 full of NaN: it must not be read in its place.
    Rounded to 16 bits once or twice, an output of at most 1 is off by 2^-8."""
    c = SmallCache(ema, [16 * 90], 2, 16, "bf16", seed=50)
    try:
        free = np.setdiff1d(np.arange(c.n_local), c.table)[0]
        c.local[[0, free]] = c.local[[free, 0]]
        c.table[c.table == 0] = free
        assert (c.local[0].view(np.uint16) == 0x7FC0).all()
        c.upload()
        gone = (66, 70)
        table = c.table.copy()
        table[0, gone] = -1, c.n_local
        n = 1 if op == "diff" else 33
        q16 = c.queries(n, 4)
        got = attend(ema, c, op, q16, [0, n], table, OUT[out]).double().cpu().numpy()
        assert np.isfinite(got).all()
        for row in {0, n // 2, n - 1}:
            ref = left_out(c, op, q16, row, 0, int(c.lens[0]) - n + row + 1, gone)
            assert np.abs(ref).max() < 1
            assert np.abs(got[row] - ref).max() < (2.0 ** -8 if out == "bf16" else 1e-4)
    finally:
        c.close()


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("lens,new,bs", [
    ([300, 0, 5], [300, 0, 5], 16),                      # several tiles of rows
    ([4000, 700], [4, 1], 16),                           # the tokens in several parts
    ([1500, 1000, 129], [40, 1000, 129], 64),
    ([1025, 2049], [1, 2049], 256),
])
@pytest.mark.parametrize("op", ["prompt", "diff-prompt"])
def test_bad_entries_of_chunks_are_counted_once(ema, op, lens, new, bs, out):
    c = SmallCache(ema, lens, 4, bs, "bf16", seed=51)
    try:
        T = sum(new)
        q16, starts = c.queries(T, 8), np.concatenate([[0], np.cumsum(new)])
        maps = 1 if op == "prompt" else 2
        q, lam = dev16(q16, "bf16"), torch.ones(4, device="cuda")
        o = torch.zeros((T, 8 // maps, maps * D), dtype=OUT[out], device="cuda")
        for places in ([(0, 0)], [(0, -1)], [(b, j) for b, n in enumerate(lens)
                                             for j in range(0, -(-n // bs), 3)]):
            table = c.table.copy()
            for b, j in places:
                table[b, j % max(1, -(-lens[b] // bs))] = -7
            bad = sum(int((table[b, :-(-n // bs)] == -7).sum()) for b, n in enumerate(lens))
            if op == "prompt":
                ema.paged_prompt_attention(c.h, q, i32(starts), i32(table), c.lens_dev, o)
            else:
                ema.paged_diff_prompt_attention(c.h, q, i32(starts), i32(table), c.lens_dev, lam, o)
            assert ema.slice_device_errors(c.h) == bad
    finally:
        c.close()


@pytest.mark.parametrize("heads", [2, 9])
@pytest.mark.parametrize("lens,bs", [([2100, 777, 40, 0], 16), ([1057], 16), ([900, 33] * 9, 32),
                                     ([1500, 64], 64), ([30] * 300, 16), ([600, 255], 256)])
def test_bad_entries_of_single_tokens_are_counted_once(ema, lens, bs, heads):
    c = SmallCache(ema, lens, 4, bs, "bf16", seed=52)
    try:
        B = len(lens)
        q, lam = dev16(c.queries(B, 4 * heads), "bf16"), torch.ones(2 * heads, device="cuda")
        o = torch.zeros((B, 2 * heads, 2 * D), device="cuda")
        for step in (1, 3, 64):
            table = c.table.copy()
            table[:, ::step] = c.n_local
            table[:, -1] = -9                            # behind every length: not looked at
            bad = sum(len(range(0, -(-n // bs), step)) for n in lens)
            ema.paged_diff_attention(c.h, q, i32(table), c.lens_dev, lam, o)
            assert ema.slice_device_errors(c.h) == bad
            if step == 1:
                assert (o == 0).all()
    finally:
        c.close()


@pytest.mark.parametrize("starts,bad", [([1, 3, 10], 1), ([0, 6, 2], 1), ([0, 12, 11], 2),
                                        ([-4, 3, 10], 1), ([0, 3, 2 ** 31 - 1], 1)])
@pytest.mark.parametrize("maps", [1, 2])
def test_bad_starts_are_counted(ema, maps, starts, bad):
    """Starts that do not begin at 0, descend or pass the rows: a request each."""
    c = SmallCache(ema, [64, 40], 2, 16, "bf16", seed=53)
    try:
        q, lam = dev16(c.queries(10, 4), "bf16"), torch.ones(2, device="cuda")
        o = torch.zeros((10, 4 // maps, maps * D), device="cuda")
        if maps == 1:
            ema.paged_prompt_attention(c.h, q, i32(starts), c.table_dev, c.lens_dev, o)
        else:
            ema.paged_diff_prompt_attention(c.h, q, i32(starts), c.table_dev, c.lens_dev, lam, o)
        assert ema.slice_device_errors(c.h) == bad
    finally:
        c.close()


@pytest.mark.parametrize("B", [100, 700])
@pytest.mark.parametrize("maps", [1, 2])
def test_bad_starts_among_many_requests_are_counted(ema, maps, B):
    c = SmallCache(ema, [3] * B, 2, 16, "bf16", seed=57)
    try:
        q, lam = dev16(c.queries(B, 4), "bf16"), torch.ones(2, device="cuda")
        o = torch.zeros((B, 4 // maps, maps * D), device="cuda")
        starts = np.arange(B + 1)
        starts[[70, 71]] = starts[[71, 70]]              # request 70 ends before it begins
        starts[B] = B + 5                                # the last one ends past the rows
        if maps == 1:
            ema.paged_prompt_attention(c.h, q, i32(starts), c.table_dev, c.lens_dev, o)
        else:
            ema.paged_diff_prompt_attention(c.h, q, i32(starts), c.table_dev, c.lens_dev, lam, o)
        assert ema.slice_device_errors(c.h) == 2
    finally:
        c.close()
