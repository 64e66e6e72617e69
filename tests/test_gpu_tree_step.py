"""Steps that draft trees, all operators together as a server uses them: tables and
masks built on the GPU, slice blocks with older tokens prefetched, the nodes' K and V
stored, attention of the trees, the touched staged copies written back, the path that
the model's choices confirm found and its tokens moved behind the older ones in
both pools -- step after step, then a decode step over what was kept. An oracle
replays the block movement; both pools are compared byte for byte."""
import numpy as np
import pytest
import torch

import oracle
import synth
from harness import TORCH_DT, Workload, oracle_mirror, rel_err
from ops_harness import assert_close, dev16, i32
from oracle import ops as oops, trees
from paper_2609_27040_amd.step import run_tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def draft(rng, n):
    p = np.maximum(np.arange(n) - 1 - rng.integers(0, 3, n), 0)
    p[:1] = -1
    return p


def grow(w, base, nodes):
    """The cache's lengths with the drafted tokens."""
    w.lens = base + nodes
    w.lens_dev.copy_(torch.from_numpy(w.lens.astype(np.int32)))


@pytest.mark.parametrize("layout,side,graph", [(0, False, False), (1, False, False),
                                               (1, True, False), (0, False, True)])
def test_trees_drafted_and_committed(layout, side, graph):
    cfg = synth.TINY.scaled(q_heads=8, kv_heads=2, dtype="bf16")
    full = np.array([130, 40, 90, 16, 260])
    w = Workload(cfg, layers=4, slice_layout=layout, staging_slots=2, lens=full, frac=0.4)
    st = oracle_mirror(w)
    rng = np.random.default_rng(8)
    dt = TORCH_DT["bf16"]
    stream = torch.cuda.Stream() if side else None
    try:
        base = np.array([100, 5, 0, 3, 190])
        for nodes in ([12, 20, 7, 0, 66], [9, 1, 30, 11, 5], [0, 0, 1, 0, 0]):
            nodes = np.array(nodes)
            grow(w, base, nodes)
            parents = [draft(rng, n) for n in nodes]
            tree = w.tree(parents, stream=stream)
            T, starts = tree.T, np.concatenate([[0], np.cumsum(nodes)])
            words = max(1, -(-nodes.max() // 64))
            flat = np.concatenate(parents)
            mask, pos, first = trees.tree_tables(flat, starts, w.lens, words)
            torch.cuda.synchronize()
            assert np.array_equal(tree.mask.cpu().numpy().view(np.uint64), mask)
            assert np.array_equal(tree.positions.cpu().numpy(), pos)
            assert np.array_equal(tree.base.cpu().numpy(), first) and (first == base).all()
            data = [[synth.random_16bit(rng, (T, h, w.D), "bf16") for h in (8, 2, 2)]
                    for _ in range(w.L)]
            dev = [[dev16(x, "bf16") for x in d] for d in data]
            outs = [torch.zeros((T, 8, w.D), dtype=dt, device="cuda") for _ in range(w.L)]
            torch.cuda.synchronize()
            if graph:
                s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=s):
                    run_tree(w, tree, lambda l: (*dev[l], outs[l]), stream=s)
                before = [v.clone() for v in (w.local_view, w.slice_view)]
                for _ in range(3):                     # the same step from the same pools
                    w.local_view.copy_(before[0])
                    w.slice_view.copy_(before[1])
                    for o in outs:
                        o.zero_()
                    torch.cuda.synchronize()
                    g.replay()
                    torch.cuda.synchronize()
            else:
                run_tree(w, tree, lambda l: (*dev[l], outs[l]), stream=stream)
            torch.cuda.synchronize()
            used = np.arange(w.maxblk)[None, :] < (-(-w.lens // w.bs))[:, None]
            for l in range(w.L):
                q, k, v = data[l]
                ref = oops.kv_tables([w.tables[l][used]], w.lens, nodes, w.maxblk, w.bs, w.n_local, T,
                                     w.staging[l % w.staging_slots][None], 10 ** 4)
                n, m = int(ref["prefetch"][2][0]), int(ref["writeback"][2][0])
                st.prefetch(ref["prefetch"][0][0, :n], ref["prefetch"][1][0, :n])
                oops.kv_store(st.local, k, v, ref["slots"][0], w.hkv, w.D, w.bs)
                want, mass = trees.tree_attention(q, starts, ref["table"][0], w.lens, mask,
                                                  st.read_block, 2, w.D, w.bs, "bf16")
                st.writeback(ref["writeback"][0][0, :m], ref["writeback"][1][0, :m])
                assert_close(outs[l], want, mass, dt, "bf16", int(w.lens.max()))
            # what a model of three tokens makes of it
            drafted, choice = rng.integers(0, 3, T), rng.integers(0, 3, T)
            path, n_path, after = w.accept(tree, i32(drafted), i32(choice), cap=5, stream=stream)
            kept = trees.tree_accept(flat, starts, drafted, choice, 5)
            w.commit(tree, path, n_path, stream=stream)
            torch.cuda.synchronize()
            for got, ref in zip((path, n_path, after), kept):
                assert np.array_equal(got.cpu().numpy(), ref)
            base = trees.kv_compact(st.local, st.slice, layout == 1, w.tables, base, kept[0], kept[1],
                                    w.hkv, w.D, w.bs)
            assert np.array_equal(w.lens, base) and np.array_equal(w.lens_dev.cpu().numpy(), base)
            assert np.array_equal(w.local_view.cpu().numpy(), st.local)
            assert np.array_equal(w.slice_view.cpu().numpy(), st.slice)
        # a decode step over what was kept
        keep = w.tables.copy()
        w.tables[:, np.arange(w.maxblk)[None, :] >= (-(-w.lens // w.bs))[:, None]] = -1
        w.restage()
        for l in range(w.L):
            w.prefetch(l)
            st.prefetch(w.pf_src[l], w.pf_dst[l])
            out = w.new_out()
            w.attention(l, out)
            ref = oracle.paged_decode_attention(w.q16, w.attn_tables[l], w.lens, st.read_block, 2,
                                                w.D, w.bs, "bf16")
            assert rel_err(out.cpu().numpy(), ref) <= 2e-3
        w.tables = keep
        from paper_2609_27040_amd import ema
        assert ema.slice_device_errors(w.h) == 0
    finally:
        w.close()


def test_parents_are_checked():
    w = Workload(synth.TINY.scaled(q_heads=8, kv_heads=2), layers=1, lens=np.array([30, 20]), frac=0.0)
    try:
        w.tree([[-1, 0], []])
        for bad in ([[0], []], [[-1, 1], []], [[-2], []], [[-1]], [[-1] * 31, []]):
            with pytest.raises(ValueError):
                w.tree(bad)
    finally:
        w.close()
