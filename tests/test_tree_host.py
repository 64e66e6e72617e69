"""The operators of include/ema_tree.h without a GPU: what the library exports, what
the entry points refuse, host-only validation, and the oracle on cases by hand."""
import ctypes
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ema_tree.h")
LIB = os.path.join(ROOT, "paper_2609_27040_amd", "lib", "libema_slice.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
D = 128
i32 = lambda a: np.array(a, np.int32)
z = lambda *s: np.zeros(s, np.int32)


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(ema_[a-z_]+)\s*\(", text)))


def test_every_operator_is_exported_and_bound():
    from paper_2609_27040_amd import ema
    names = declared()
    assert len(names) == 5
    for n in names:
        assert hasattr(ema._lib, n) and hasattr(ema, n[len("ema_"):]), n


def test_a_null_handle_is_refused():
    from paper_2609_27040_amd import ema
    n = None
    calls = {
        "ema_tree_tables": (n, n, n, n, 0, 0, n, 1, n, n, n),
        "ema_paged_tree_workspace": (n, 0, 0, 0, 0, n),
        "ema_paged_tree_attention": (n, n, 0, n, n, n, n, 1, 0, 0, 0, 0, 0.0, n, 2, n, 0, n),
        "ema_tree_accept": (n, n, n, n, n, n, 0, 0, 1, n, n, n, n),
        "ema_kv_compact": (n, n, n, n, n, 1, 0, 0, 0, n, n),
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


class _Mask:
    def __init__(self, *shape):
        self.shape = shape


class _Q:
    def __init__(self, rows, heads):
        self.shape = (rows, heads, D)


def test_trees_are_validated_on_the_host(host):
    ema, h = host
    f = lambda parents, starts, lens, words=1: ema.tree_tables(
        h, i32(parents), i32(starts), i32(lens), _Mask(len(parents), words))
    f([-1, 0, 1, -1, -1], [0, 3, 5], [3, 9])
    f([], [0, 0], [4])
    f([-1, 7], [0, 1], [4])                                            # a row of no request
    f([-1] * 65, [0, 65], [70], 2)
    for bad in (([0], [0, 1], [4]), ([-2], [0, 1], [4]), ([-1, 1], [0, 2], [4]),
                ([-1, 0], [0, 2], [1]),                                # more nodes than tokens
                ([-1, -1], [1, 2], [4]), ([-1, -1], [0, 3], [4]), ([-1, -1], [0, 2, 1], [4, 4]),
                ([-1, -1], [0, 5, 2], [9, 9]),
                ([-1] * 65, [0, 65], [70]), ([-1], [0, 1], [4], 17), ([-1], [0, 1], [4], 0)):
        refused(ema, f, *bad)


def test_paths_are_validated_on_the_host(host):
    ema, h = host

    def f(parents, starts, cap=3, B=None):
        B = len(starts) - 1 if B is None else B
        n = len(parents)
        ema.tree_accept(h, i32(parents), i32(starts), z(n), z(n), z(B, cap), z(B), z(B))

    f([-1, 0, -1], [0, 2, 3])
    f([-1] * 1024, [0, 1024])
    for bad in (([0], [0, 1]), ([-1, -2], [0, 2]), ([-1], [0, 2]), ([-1] * 1025, [0, 1025]),
                ([-1], [0, 1], 0), ([-1], [0, 1], 3, 2)):
        refused(ema, f, *bad)


def test_lists_are_validated_on_the_host(host):
    ema, h = host

    def f(table, base, keep, n, lens=None):
        ema.kv_compact(h, i32(table), i32(base), i32(keep), i32(n), new_lens=lens)

    t = [[[0, 1, -1], [13, 3, 17]]]                                    # local and slice blocks
    f(t, [16, 0], [[0, 3, 4], [1, 20, 47]], [3, 3], z(2))
    f(t, [16, 0], [[0, 3, -9], [1, 20, 99]], [2, 0])                   # behind the counts: not looked at
    f([[[-1, 1, -1], [13, 3, 17]]], [5, 0], [[0, 1, 2], [1, 20, 47]], [3, 3])   # nothing moves there
    bad = [([-1, 0], [[0, 1, 2], [0, 1, 2]], [3, 3]), ([0, 0], [[0, 1, 2], [0, 1, 2]], [4, 3]),
           ([0, 0], [[0, 1, 2], [0, 1, 2]], [-1, 3]), ([0, 0], [[0, 3, 3], [0, 1, 2]], [3, 3]),
           ([0, 0], [[0, 4, 3], [0, 1, 2]], [3, 3]), ([0, 0], [[-1, 1, 2], [0, 1, 2]], [3, 3]),
           ([0, 1], [[0, 1, 2], [0, 1, 47]], [3, 3]),                  # past the table
           ([30, 0], [[0, 1, 2], [0, 1, 2]], [3, 3])]                  # nothing moves: see below
    for a in bad[:-1]:
        refused(ema, f, t, *a)
    f(t, *bad[-1])
    refused(ema, f, t, [30, 0], [[0, 1, 3], [0, 1, 2]], [3, 3])        # its blocks are not there
    refused(ema, f, [[[18, 1, 2], [0, 1, 2]]], [0, 0], [[1, 2, 3], [0, 1, 2]], [3, 3])
    refused(ema, f, t, [0], [[0, 1, 2], [0, 1, 2]], [3, 3])            # arrays that do not fit
    refused(ema, f, t, [0, 0], [[0, 1, 2], [0, 1, 2]], [3])
    refused(ema, f, t, [0, 0], [[0, 1, 2], [0, 1, 2]], [3, 3], z(1))
    refused(ema, f, t[0], [0, 0], [[0, 1, 2], [0, 1, 2]], [3, 3])
    lib, p = ema._lib, z(4).ctypes.data
    for L, B, width, cap in ((0, 1, 1, 1), (65536, 1, 1, 1), (1, -1, 1, 1), (1, 65536, 1, 1),
                             (1, 1, -1, 1), (1, 1, 1, -1), (1, 1, 1 << 27, 1)):
        assert lib.ema_kv_compact(h, p, p, p, p, L, B, width, cap, None, None) == ema.ERR_INVAL
    for args in ((None, p, p, p), (p, None, p, p), (p, p, None, p), (p, p, p, None)):
        assert lib.ema_kv_compact(h, *args, 1, 1, 1, 1, None, None) == ema.ERR_INVAL
    assert lib.ema_kv_compact(h, None, None, None, None, 1, 0, 0, 0, None, None) == ema.OK


def test_attention_is_validated_on_the_host(host):
    ema, h = host

    def f(starts, table, lens, rows=8, heads=4, words=1, masks=None):
        ema.paged_tree_attention(h, _Q(rows, heads), i32(starts), i32(table), i32(lens),
                                 _Mask(rows if masks is None else masks, words), None)

    t = [[0, 1, -1], [2, 3, 4]]
    f([0, 3, 8], t, [20, 48])
    f([0, 0, 8], [[-1, -1, -1], [2, 3, 4]], [20, 48])                  # no rows: not read
    for a in (([1, 3, 8], t, [20, 48]), ([0, 3, 9], t, [20, 48]), ([0, 5, 3], t, [20, 48]),
              ([0, 3, 8], t, [2, 48]), ([0, 3, 8], t, [20, 49]), ([0, 3, 8], t, [-1, 48]),
              ([0, 3, 8], [[0, 12, -1], [2, 3, 4]], [20, 48])):
        refused(ema, f, *a)
    for kw in (dict(heads=3), dict(heads=0), dict(words=0), dict(words=17)):
        refused(ema, f, [0, 3, 8], t, [20, 48], **kw)
    n = ctypes.c_size_t()
    size = ema._lib.ema_paged_tree_workspace
    for tokens, batch, heads, width in ((-1, 1, 4, 1), (1, -1, 4, 1), (1, 65536, 4, 1),
                                        (1, 1, 4098, 1), (1, 1, 4, (1 << 26) + 1),
                                        (1 << 27, 1, 4, 1)):
        assert size(h, tokens, batch, heads, width, ctypes.byref(n)) == ema.ERR_INVAL
    assert size(h, 5, 1, 4, 1, None) == ema.ERR_INVAL
    assert size(h, 65535, 65535, 4, 1 << 15, ctypes.byref(n)) == ema.ERR_INVAL   # tiles: 32 bits
    assert size(h, 65535, 65535, 4, 1 << 14, ctypes.byref(n)) == ema.OK


def test_arrays_of_another_rank_or_type(host):
    ema, h = host
    ok = dict(parents=z(1) - 1, query_start=i32([0, 1]), seq_lens=i32([1]), mask=_Mask(1, 1))
    ema.tree_tables(h, **ok)
    for bad in (dict(parents=z(1, 1)), dict(query_start=z(1, 2)), dict(query_start=z(0)),
                dict(seq_lens=z(2)), dict(mask=_Mask(1)), dict(mask=_Mask(2, 1)),
                dict(parents=np.array([-1])), dict(positions=z(2)), dict(base=z(2))):
        refused(ema, ema.tree_tables, h, **{**ok, **bad})
    ok = dict(parents=z(1) - 1, query_start=i32([0, 1]), drafted=z(1), choice=z(1), path=z(1, 2),
              n_path=z(1), next_token=z(1))
    ema.tree_accept(h, **ok)
    for bad in (dict(path=z(1)), dict(path=z(2, 2)), dict(drafted=z(2)), dict(choice=z(0)),
                dict(n_path=z(2)), dict(next_token=z(2)), dict(root_choice=z(2)),
                dict(drafted=np.zeros(1, np.int64))):
        refused(ema, ema.tree_accept, h, **{**ok, **bad})
    refused(ema, ema.kv_compact, h, z(1, 1, 1), z(1), z(1), z(1))


def test_the_oracle_by_hand():
    from oracle import trees
    #  0 - 1 - 3    4 (a root)
    #    \ 2 - 5
    parents, starts = [-1, 0, 0, 1, -1, 2], [0, 6]
    mask, pos, base = trees.tree_tables(parents, starts, [16], 1)
    assert mask[:, 0].tolist() == [1, 3, 5, 11, 16, 37]
    assert pos.tolist() == [10, 11, 11, 12, 10, 12] and base.tolist() == [10]
    drafted, choice = [7, 8, 9, 8, 7, 1], [9, 0, 1, 0, 0, 4]
    path, n, after = trees.tree_accept(parents, starts, drafted, choice, 4)
    assert path.tolist() == [[0, 2, 5, -1]] and n.tolist() == [3] and after.tolist() == [4]
    path, n, after = trees.tree_accept(parents, starts, drafted, choice, 2, [7])   # 4 has 7 too
    assert path.tolist() == [[0, 2]] and after.tolist() == [1]
    path, n, after = trees.tree_accept(parents, starts, drafted, choice, 2, [3])
    assert path.tolist() == [[-1, -1]] and n.tolist() == [0] and after.tolist() == [3]
    # tokens 1, 2, 3 <- 2, 3, 17 of a request of two blocks, the second in the slice
    local, far = (np.arange(3 * 8192, dtype=np.uint16).view(np.uint8).reshape(3, -1) for _ in "lf")
    local, far = local.copy(), far[:2].copy()
    before = [x.view(np.uint16).reshape(len(x), 2, -1).copy() for x in (local, far)]
    lens = trees.kv_compact(local, far, True, np.array([[[1, 4]]]), [1], [[1, 2, 16]], [3], 2, 128,
                            16)
    assert lens.tolist() == [4]
    K, V = (local.view(np.uint16).reshape(3, 2, -1)[1, i] for i in (0, 1))
    k0, v0 = before[0][1]
    for head in (0, 1):
        rows = K.reshape(2, 16, 128)[head]
        assert (rows[1:3] == k0.reshape(2, 16, 128)[head, 2:4]).all()
        assert (rows[3] == before[1][1, 0].reshape(16, 2, 128)[1, head]).all()
        cols = V.reshape(2, 128, 16)[head]
        assert (cols[:, 1:3] == v0.reshape(2, 128, 16)[head][:, 2:4]).all()
        assert (cols[:, 3] == before[1][1, 1].reshape(16, 2, 128)[1, head]).all()


def test_the_attention_oracle_of_a_chain_is_the_causal_one():
    import synth
    from oracle import ops, trees
    rng = np.random.default_rng(0)
    blocks = synth.random_16bit(rng, (5, 2 * 2 * 16 * D), "bf16").view(np.uint8)
    table, lens, starts = np.array([[3, 0], [4, 2]]), [25, 32], [0, 4, 9]
    q = synth.random_16bit(rng, (9, 4, D), "bf16")
    chain = np.concatenate([np.arange(4), np.arange(5)]) - 1
    mask = trees.tree_tables(chain, starts, lens, 1)[0]
    a = trees.tree_attention(q, starts, table, lens, mask, lambda u: blocks[u], 2, D, 16, "bf16")
    b = ops.prompt_attention(q, starts, table, lens, lambda u: blocks[u], 2, D, 16, "bf16")
    assert np.allclose(a, b, rtol=1e-12, atol=0)
