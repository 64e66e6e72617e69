"""Calls on the default stream while another one is current: stream 0 is the default stream
for memory and waits too."""
import numpy as np
import pytest
import torch

import synth
from harness import Workload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


def test_torch_streams(ema):
    side = torch.cuda.Stream()
    assert ema.torch_stream(0) == torch.cuda.default_stream()
    assert ema.torch_stream(torch.cuda.default_stream()) == torch.cuda.default_stream()
    assert ema.torch_stream(side).cuda_stream == side.cuda_stream
    assert ema.torch_stream(side.cuda_stream).cuda_stream == side.cuda_stream
    with torch.cuda.stream(side):
        assert ema.torch_stream(None).cuda_stream == side.cuda_stream


def test_a_workspace_on_the_default_stream(ema):
    """Its memory comes from the default stream's, and goes back there."""
    n, device = 1 << 20, torch.device("cuda", 0)
    with torch.cuda.stream(torch.cuda.Stream()):
        ws, at, _ = ema._scratch(n, None, 0, device)
        del ws
    assert torch.empty(n, dtype=torch.uint8, device=device).data_ptr() == at


def test_a_chunk_built_on_the_default_stream(ema):
    cfg = synth.TINY.scaled(q_heads=8, kv_heads=2, dtype="bf16")
    w = Workload(cfg, layers=3, staging_slots=2, lens=np.array([90, 33]), frac=0.5)
    try:
        want = w.chunk([40, 33])
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
            got = w.chunk([40, 33], stream=torch.cuda.default_stream())
        torch.cuda.synchronize()
        for a, b in ((want.block_table, got.block_table), (want.slots, got.slots),
                     (want.starts, got.starts), *zip(want.prefetch, got.prefetch),
                     *zip(want.writeback, got.writeback)):
            assert torch.equal(a, b)
    finally:
        w.close()
