"""The operators of include/ema_ops.h without a GPU: what the library exports,
what the entry points refuse, and host-only validation."""
import ctypes
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ema_ops.h")
LIB = os.path.join(ROOT, "paper_2609_27040_amd", "lib", "libema_slice.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
D = 128


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(ema_[a-z_]+)\s*\(", text)))


def test_every_operator_is_exported_and_bound():
    from paper_2609_27040_amd import ema
    names = declared()
    assert len(names) == 9
    for n in names:
        assert hasattr(ema._lib, n) and hasattr(ema, n[len("ema_"):]), n


def test_a_null_handle_is_refused():
    from paper_2609_27040_amd import ema
    z = None
    calls = {
        "ema_kv_tables_workspace": (z, z, z),
        "ema_kv_tables": (z, z, z, 0, z),
        "ema_kv_store": (z, z, 0, z, 0, z, 0, z),
        "ema_paged_prompt_workspace": (z, 0, 0, 0, 0, z),
        "ema_paged_prompt_attention": (z, z, 0, z, z, z, 0, 0, 0, 0, 0.0, z, 2, z, 0, z),
        "ema_paged_diff_workspace": (z, 0, 0, 0, z),
        "ema_paged_diff_attention": (z, z, 0, z, z, 0, 0, 0, 0.0, z, z, 0.0, z, 2, z, 0, z),
        "ema_paged_diff_prompt_workspace": (z, 0, 0, 0, 0, z),
        "ema_paged_diff_prompt_attention": (z, z, 0, z, z, z, 0, 0, 0, 0, 0.0, z, z, 0.0, z, 2, z,
                                            0, z),
    }
    assert set(calls) == set(declared())
    for name, args in calls.items():
        assert getattr(ema._lib, name)(*args) == ema.ERR_INVAL, name
        assert ema.last_error(), name


@pytest.fixture
def host():
    from paper_2609_27040_amd import ema
    bb = 2 * 16 * 2 * D * 2
    h = ema.slice_create(2, D, 16, "bf16", 0, 12 * bb, 6 * bb, host_only=True)
    yield ema, h
    ema.slice_destroy(h)


def refused(ema, fn, *a, **kw):
    with pytest.raises(ema.EmaError) as e:
        fn(*a, **kw)
    assert e.value.code == ema.ERR_INVAL
    return str(e.value)


def tables(ema, h, ids, lens, new, width=3, n_slots=64, staging=None, cap=8):
    z = lambda *s: np.zeros(s, np.int32)
    ids = np.asarray(ids, np.int32)
    L, B = ids.shape[0], len(lens)
    kw = {}
    if staging is not None:
        staging = np.asarray(staging, np.int32)
        n = staging.shape[1]
        kw = dict(staging=staging, prefetch=(z(L, n), z(L, n), z(L)),
                  writeback=(z(L, cap), z(L, cap), z(L)))
    ema.kv_tables(h, ids, np.asarray(lens, np.int32), np.asarray(new, np.int32), z(L, B, width),
                  z(L, n_slots), z(B + 1), **kw)


def test_tables_are_validated_on_the_host(host):
    ema, h = host
    tables(ema, h, [[0, 1, 2]], [20, 5], [1, 5])
    tables(ema, h, [[0, 12, 2]], [20, 5], [1, 5], staging=[[3, 4]])
    bad = [
        dict(ids=[[0, 1, 2]], lens=[49, 5], new=[1, 5]),                 # past the table
        dict(ids=[[0, 1, 2]], lens=[-1, 5], new=[0, 5]),
        dict(ids=[[0, 1, 2]], lens=[20, 5], new=[21, 5]),                # more new than tokens
        dict(ids=[[0, 1, 2]], lens=[20, 5], new=[-1, 5]),
        dict(ids=[[0, 1]], lens=[20, 5], new=[1, 5]),                    # too few ids
        dict(ids=[[0, 18, 2]], lens=[20, 5], new=[1, 5]),                # outside both pools
        dict(ids=[[0, -1, 2]], lens=[20, 5], new=[1, 5]),
        dict(ids=[[0, 1, 2]], lens=[20, 5], new=[1, 5], n_slots=5),
        dict(ids=[[0, 12, 2]], lens=[20, 5], new=[1, 5]),                # a new token in the slice
        dict(ids=[[12, 13, 2]], lens=[20, 5], new=[1, 5], staging=[[3]]),
        dict(ids=[[0, 12, 2]], lens=[20, 5], new=[1, 5], staging=[[12]]),
        dict(ids=[[0, 12, 13]], lens=[20, 5], new=[1, 5], staging=[[3, 4]], cap=1),
    ]
    for kw in bad:
        refused(ema, tables, ema, h, **kw)


def test_tables_of_bad_shapes(host):
    ema, h = host
    refused(ema, tables, ema, h, [[0]], [1, 1], [1])                     # new_lens too short
    a = ema.KVTablesArgs(layers=1, batch=1, max_blocks=0)
    n = ctypes.c_size_t()
    assert ema._lib.ema_kv_tables_workspace(h, ctypes.byref(a), ctypes.byref(n)) == ema.ERR_INVAL
    a = ema.KVTablesArgs(layers=1, batch=65536, max_blocks=65536)        # 2^31 tokens and more
    assert ema._lib.ema_kv_tables_workspace(h, ctypes.byref(a), ctypes.byref(n)) == ema.ERR_INVAL
    a = ema.KVTablesArgs(layers=-1, batch=1, max_blocks=1)
    assert ema._lib.ema_kv_tables_workspace(h, ctypes.byref(a), ctypes.byref(n)) == ema.ERR_INVAL


def test_slots_are_validated_on_the_host(host):
    ema, h = host
    ema.kv_store(h, None, None, [0, 5, -1, 12 * 16 - 1, -1])
    for slots in ([12 * 16], [-2], [3, 4, 3]):
        refused(ema, ema.kv_store, h, None, None, slots)
    lib = ema._lib
    one = np.zeros(1, np.int32)
    for ks, vs in ((255, 256), (256, 252), (260, 256)):                  # strides
        assert lib.ema_kv_store(h, None, ks, None, vs, one.ctypes.data, 1, None) == ema.ERR_INVAL
    assert lib.ema_kv_store(h, None, 256, None, 256, None, 1, None) == ema.ERR_INVAL
    assert lib.ema_kv_store(h, None, 256, None, 256, None, -1, None) == ema.ERR_INVAL
    assert lib.ema_kv_store(h, None, 0, None, 0, None, 0, None) == ema.OK


class _Q:
    def __init__(self, rows, heads):
        self.shape = (rows, heads, D)


@pytest.mark.parametrize("diff", [False, True])
def test_attention_is_validated_on_the_host(host, diff):
    ema, h = host

    def call(starts, table, lens, rows=8, heads=4, **kw):
        table = np.asarray(table, np.int32)
        if diff:
            ema.paged_diff_prompt_attention(h, _Q(rows, heads), np.asarray(starts), table, lens,
                                            None, None, **kw)
        else:
            ema.paged_prompt_attention(h, _Q(rows, heads), np.asarray(starts), table, lens, None,
                                       **kw)

    t = [[0, 1, -1], [2, 3, 4]]
    call([0, 3, 8], t, [20, 48])
    call([0, 0, 8], [[-1, -1, -1], [2, 3, 4]], [20, 48])                 # no rows: not read
    for a in (([1, 3, 8], t, [20, 48]), ([0, 3, 9], t, [20, 48]), ([0, 5, 3], t, [20, 48]),
              ([0, 3, 8], t, [2, 48]), ([0, 3, 8], t, [20, 49]), ([0, 3, 8], t, [-1, 48]),
              ([0, 3, 8], [[0, 12, -1], [2, 3, 4]], [20, 48]),
              ([0, 3, 8], [[0, -1, -1], [2, 3, 4]], [20, 48])):
        refused(ema, call, *a)
    refused(ema, call, [0, 3, 8], t, [20, 48], heads=3)
    refused(ema, call, [0, 3, 8], t, [20, 48], heads=0)


def test_single_tokens_and_odd_kv_heads(host):
    ema, h = host
    f = lambda rows, table, lens: ema.paged_diff_attention(
        h, _Q(rows, 4), np.asarray(table, np.int32), lens, None, None)
    f(2, [[0, 1], [2, -1]], [17, 16])
    refused(ema, f, 3, [[0, 1], [2, -1]], [17, 16])
    refused(ema, f, 2, [[0, 1], [2, -1]], [17, 17])
    refused(ema, f, 2, [[0, 1], [2, -1]], [33, 1])
    odd = ema.slice_create(3, D, 16, "bf16", 0, 1 << 20, 0, host_only=True)
    try:
        assert "pair" in refused(ema, ema.paged_diff_attention, odd, _Q(1, 6),
                                 np.zeros((1, 1), np.int32), [1], None, None)
        ema.paged_prompt_attention(odd, _Q(1, 6), [0, 1], np.zeros((1, 1), np.int32), [1], None)
    finally:
        ema.slice_destroy(odd)


def test_single_tokens_take_16_query_heads_per_kv_head(host):
    ema, h = host
    table = np.zeros((1, 1), np.int32)
    ema.paged_diff_attention(h, _Q(1, 32), table, [1], None, None)
    assert "16" in refused(ema, ema.paged_diff_attention, h, _Q(1, 34), table, [1], None, None)
    n = ctypes.c_size_t()
    assert ema._lib.ema_paged_diff_workspace(h, 1, 34, 1, ctypes.byref(n)) == ema.ERR_INVAL
    ema.paged_diff_prompt_attention(h, _Q(1, 34), [0, 1], table, [1], None, None)


def test_sizes_past_the_limits(host):
    ema, h = host
    n = ctypes.c_size_t()
    size = ema._lib.ema_paged_prompt_workspace
    for tokens, batch, heads, width in ((-1, 1, 4, 1), (1, -1, 4, 1), (1, 65536, 4, 1),
                                        (1, 1, 4098, 1), (1, 1, 4, (1 << 26) + 1),
                                        (1 << 29, 1, 4, 1)):
        assert size(h, tokens, batch, heads, width, ctypes.byref(n)) == ema.ERR_INVAL
    assert size(h, 5, 1, 4, 1, None) == ema.ERR_INVAL
    diff = ema._lib.ema_paged_diff_prompt_workspace
    for f in (size, diff):                             # rows of the output: 32 bits
        assert f(h, 1 << 27, 1, 4, 1, ctypes.byref(n)) == ema.ERR_INVAL
        assert f(h, (1 << 27) - 1, 1, 4, 1, ctypes.byref(n)) == ema.OK
    single = ema._lib.ema_paged_diff_workspace         # tiles of all requests: 32 bits
    assert single(h, 65535, 4, 1 << 17, ctypes.byref(n)) == ema.ERR_INVAL
    assert single(h, 65535, 4, 1 << 15, ctypes.byref(n)) == ema.OK
    one = np.zeros(1, np.int32)
    assert ema._lib.ema_kv_store(h, None, 256, None, 256, one.ctypes.data, 1 << 29,
                                 None) == ema.ERR_INVAL
    a = ema.KVTablesArgs(layers=0, batch=1, max_blocks=1)
    assert ema._lib.ema_kv_tables_workspace(h, ctypes.byref(a), ctypes.byref(n)) == ema.ERR_INVAL


def test_the_table_oracle_on_a_case_by_hand():
    from oracle import ops
    # request 0: blocks 0 and slice 20, tokens 18 and 19 new; request 1: 2, slice 21
    # and 5, tokens 16..32 new, so nothing older is in 21
    r = ops.kv_tables([[0, 20, 2, 21, 5]], [20, 33], [2, 17], 3, 16, 10, 21, np.array([[7, 8]]), 3)
    assert r["canon"].tolist() == [[[0, 20, -1], [2, 21, 5]]]
    assert r["table"].tolist() == [[[0, 7, -1], [2, 8, 5]]]
    assert r["starts"].tolist() == [0, 2, 19]
    assert r["slots"].tolist() == [[114, 115, *range(128, 144), 80, -1, -1]]
    assert [x.tolist() for x in r["prefetch"]] == [[[20, -1]], [[7, -1]], [1]]
    assert [x.tolist() for x in r["writeback"]] == [[[7, 8, -1]], [[20, 21, -1]], [2]]


def test_the_attention_oracle_against_the_decode_oracle():
    import oracle
    import synth
    from oracle import ops
    rng = np.random.default_rng(0)
    H, bs = 2, 16
    blocks = synth.random_16bit(rng, (5, 2 * H * bs * D), "bf16").view(np.uint8)
    table, lens = np.array([[3, 0], [4, 2]]), [25, 32]
    q = synth.random_16bit(rng, (2, 4, D), "bf16")
    one = oracle.paged_decode_attention(q, table, lens, lambda u: blocks[u], H, D, bs, "bf16")
    got, mass = ops.prompt_attention(q, [0, 1, 2], table, lens, lambda u: blocks[u], H, D, bs,
                                     "bf16")
    assert np.allclose(got, one, rtol=1e-12, atol=0) and (mass >= np.abs(got)).all()
    # a second map of weight zero leaves the first, over both heads' values
    diff, _ = ops.prompt_attention(q, [0, 1, 2], table, lens, lambda u: blocks[u], H, D, bs,
                                   "bf16", lam=np.zeros(2))
    two = q.copy()
    two[:, 1], two[:, 2], two[:, 3] = q[:, 0], q[:, 0], q[:, 0]
    first, _ = ops.prompt_attention(two[:, [0, 1]], [0, 1, 2], table, lens, lambda u: blocks[u], H,
                                    D, bs, "bf16")
    assert np.allclose(diff[:, 0, :D], first[:, 0])
    # and both maps the same cancel at weight one
    same = np.stack([q[:, 0], q[:, 0]], axis=1)
    for u in range(5):
        e = blocks[u].view(np.uint16).reshape(2, H, -1)
        e[0, 1] = e[0, 0]
    zero, _ = ops.prompt_attention(same, [0, 1, 2], table, lens, lambda u: blocks[u], H, D, bs,
                                   "bf16", lam=np.ones(1))
    assert np.abs(zero).max() < 1e-15
