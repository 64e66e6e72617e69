"""Attention of chunks where a token's query heads of a KV head are more than a workgroup's
rows (256 plain, 128 and, for 32-bit outputs, 64 differential): every row is written."""
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


@pytest.mark.parametrize("lens,new", [
    ([1], [1]),
    ([30, 1, 0, 90], [1, 1, 0, 5]),
    ([2500, 40], [2, 1]),                                # the tokens in several parts
])
@pytest.mark.parametrize("maps,out,heads", [(1, "bf16", 257), (1, "f32", 520), (2, "bf16", 129),
                                            (2, "f32", 65), (2, "f32", 300)])
def test_a_token_in_several_tiles(ema, lens, new, maps, out, heads):
    c = SmallCache(ema, lens, maps, 16, "bf16", seed=heads)
    try:
        check_attention(ema, c, new, maps * heads, out, maps, pad=1)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()


@pytest.mark.parametrize("maps,out,heads", [(1, "bf16", 300), (2, "f32", 100)])
def test_many_chunks_of_tokens_in_several_tiles(ema, maps, out, heads):
    c = SmallCache(ema, [33, 20, 7], maps, 16, "bf16", seed=heads)
    try:
        check_attention(ema, c, [33, 9, 1], maps * heads, out, maps)
    finally:
        c.close()
