"""Output types of the attention operators that are taken and refused, on a host-only handle."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_27040_amd", "lib", "libema_slice.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")


def test_output_types():
    from paper_2609_27040_amd import ema
    h = ema.slice_create(2, 128, 16, "bf16", 0, 1 << 20, 0, host_only=True)
    try:
        for code in (0, 1, 2, 3, -1, 0x80, 0x200):
            for full in (0, ema.FULL_WEIGHTS):
                rc = [ema._lib.ema_paged_prompt_attention(h, None, 0, None, None, None, 0, 0, 4, 0,
                                                          0.0, None, code | full, None, 0, None),
                      ema._lib.ema_paged_diff_attention(h, None, 0, None, None, 0, 4, 0, 0.0, None,
                                                        None, 0.0, None, code | full, None, 0, None)]
                assert rc == [ema.OK if code in (0, 1, 2) else ema.ERR_INVAL] * 2, (code, full)
    finally:
        ema.slice_destroy(h)
