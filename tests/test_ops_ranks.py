"""Arrays of another rank than documented are refused with the library's own error."""
import os

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_27040_amd", "lib", "libema_slice.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
z = lambda *s: np.zeros(s, np.int32)


@pytest.fixture
def host():
    from paper_2609_27040_amd import ema
    h = ema.slice_create(2, 128, 16, "bf16", 0, 1 << 20, 1 << 20, host_only=True)
    yield ema, h
    ema.slice_destroy(h)


def test_tables(host):
    ema, h = host
    lists = lambda n: (z(1, n), z(1, n), z(1))
    ok = dict(block_ids=z(1, 1), seq_lens=z(1), new_lens=z(1), block_table=z(1, 1, 1),
              slot_map=z(1, 1), query_start=z(2), staging=z(1, 1), prefetch=lists(1),
              writeback=lists(1))
    ema.kv_tables(h, **ok)
    for bad in (dict(block_table=z(1, 1)), dict(block_ids=z(1)), dict(block_ids=z()),
                dict(slot_map=z()), dict(staging=z(1)), dict(prefetch=lists(1)[:2]),
                dict(writeback=()), dict(writeback=(z(), z(), z(1)))):
        with pytest.raises(ema.EmaError) as e:
            ema.kv_tables(h, **{**ok, **bad})
        assert e.value.code == ema.ERR_INVAL, bad


class _Q:
    def __init__(self, *shape):
        self.shape = shape


def test_queries_and_tables_of_attention(host):
    ema, h = host
    for shape in ((), (1,), (1, 2)):
        with pytest.raises(ema.EmaError):
            ema.paged_prompt_attention(h, _Q(*shape), z(2), z(1, 1), z(1), None)
        with pytest.raises(ema.EmaError):
            ema.paged_diff_attention(h, _Q(*shape), z(1, 1), z(1), None, None)
    with pytest.raises(ema.EmaError):
        ema.paged_prompt_attention(h, _Q(1, 2, 128), z(2), z(1), z(1), None)
