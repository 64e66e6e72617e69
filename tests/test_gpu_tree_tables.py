"""Steps of drafted trees in a cache whose blocks come and go as a server's do: allocated
when a step needs them, given to another sequence after a restart, moved between the pools
before a path is kept. An oracle replays the block movement; both pools are compared byte
for byte."""
import numpy as np
import pytest
import torch

import synth
from harness import Workload, oracle_mirror
from ops_harness import dev16, i32
from oracle import ops as oops, trees
from paper_2609_27040_amd import ema
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


class Server:
    """A cache, its oracle, and the blocks that its sequences have."""

    def __init__(self, layout, side, **kw):
        cfg = synth.TINY.scaled(q_heads=4, kv_heads=2, dtype="bf16")
        self.w = w = Workload(cfg, layers=3, slice_layout=layout, staging_slots=2, stage_n=40,
                              lens=np.array([300, 40, 90, 170]), frac=0.4, extra_local=20,
                              extra_slice=20, **kw)
        self.st, self.rng = oracle_mirror(w), np.random.default_rng(layout)
        self.nhd, self.stream = layout == 1, torch.cuda.Stream() if side else None
        wide = np.full((w.L, w.B, w.maxblk + 5), -1, np.int64)
        wide[:, :, :w.maxblk] = w.tables
        w.tables = wide
        self.base = np.zeros(w.B, np.int64)

    def free(self, b, first):
        """Sequence b's blocks from logical block `first` on."""
        ids = self.w.tables[:, b, first:]
        gone = ids[ids >= 0]
        ema.slice_free_blocks(self.w.h, gone)
        self.st.free_blocks(gone)
        ids[:] = -1

    def alloc(self, pool, owners):
        ids = ema.slice_alloc_blocks(self.w.h, pool, owners)
        assert np.array_equal(ids, self.st.alloc_blocks(pool, owners))
        return ids

    def pool(self):
        return ema.POOL_SLICE if self.rng.random() < 0.5 else ema.POOL_LOCAL

    def grow(self, nodes):
        """Lengths with the nodes, and the blocks that they need."""
        w = self.w
        w.lens = self.base + nodes
        w.lens_dev.copy_(torch.from_numpy(w.lens.astype(np.int32)))
        for b, n in enumerate(-(-w.lens // w.bs)):
            for j in range(n):
                if w.tables[0, b, j] < 0:
                    for l in range(w.L):
                        w.tables[l, b, j] = self.alloc(self.pool(), np.array([b]))[0]

    def migrate(self, l, b, j):
        """Layer l's logical block j of sequence b to the other pool."""
        w = self.w
        src = w.tables[l, b, j]
        dst = self.alloc(ema.POOL_LOCAL if src >= w.n_local else ema.POOL_SLICE, np.array([b]))
        ema.slice_migrate(w.h, i32([src]), i32(dst), stream=self.stream)
        self.st.migrate(np.array([src]), dst)
        torch.cuda.synchronize()
        ema.slice_free_blocks(w.h, np.array([src]))
        self.st.free_blocks(np.array([src]))
        w.tables[l, b, j] = dst[0]

    def step(self, nodes, cap=5, before_commit=lambda: None):
        """Trees of `nodes` drafted, stored and committed."""
        w, st, rng = self.w, self.st, self.rng
        nodes = np.array(nodes)
        self.grow(nodes)
        parents = [draft(rng, n) for n in nodes]
        flat, starts = np.concatenate(parents), np.concatenate([[0], np.cumsum(nodes)])
        tree = w.tree(parents, stream=self.stream)
        data = [[synth.random_16bit(rng, (tree.T, h, w.D), "bf16") for h in (4, 2, 2)]
                for _ in range(w.L)]
        dev = [[dev16(x, "bf16") for x in d] for d in data]
        out = torch.empty((tree.T, 4, w.D), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        run_tree(w, tree, lambda l: (*dev[l], out), stream=self.stream)
        torch.cuda.synchronize()
        used = np.arange(w.tables.shape[2])[None, :] < (-(-w.lens // w.bs))[:, None]
        for l in range(w.L):
            ref = oops.kv_tables([w.tables[l][used]], w.lens, nodes, w.tables.shape[2], w.bs,
                                 w.n_local, tree.T, w.staging[l % w.staging_slots][None], 10 ** 4)
            n, m = int(ref["prefetch"][2][0]), int(ref["writeback"][2][0])
            st.prefetch(ref["prefetch"][0][0, :n], ref["prefetch"][1][0, :n])
            oops.kv_store(st.local, *data[l][1:], ref["slots"][0], w.hkv, w.D, w.bs)
            st.writeback(ref["writeback"][0][0, :m], ref["writeback"][1][0, :m])
        before_commit()
        drafted, choice = rng.integers(0, 2, tree.T), rng.integers(0, 2, tree.T)
        drafted[starts[:-1][nodes > 1] + 1] = 7        # never chosen: paths leave tokens out
        path, n_path, after = w.accept(tree, i32(drafted), i32(choice), cap=cap, stream=self.stream)
        w.commit(tree, path, n_path, stream=self.stream)
        torch.cuda.synchronize()
        kept = trees.tree_accept(flat, starts, drafted, choice, path.shape[1])
        for got, want in zip((path, n_path, after), kept):
            assert np.array_equal(got.cpu().numpy(), want)
        self.base = trees.kv_compact(st.local, st.slice, self.nhd, w.tables, self.base, kept[0],
                                     kept[1], w.hkv, w.D, w.bs)
        assert np.array_equal(w.lens, self.base)
        assert np.array_equal(w.lens_dev.cpu().numpy(), self.base)
        for view, want, name in ((w.local_view, st.local, "local"), (w.slice_view, st.slice, "slice")):
            same = (view.cpu().numpy() == want).all(axis=1)
            assert same.all(), (name, np.flatnonzero(~same))
        assert ema.slice_device_errors(w.h) == 0
        return kept[1]


@pytest.mark.parametrize("layout,side", [(0, False), (1, False), (1, True)])
def test_blocks_that_come_and_go_between_commits(layout, side):
    s = Server(layout, side)
    w = s.w
    try:
        s.base = np.array([250, 16, 77, 100])
        for b, n in enumerate(-(-s.base // w.bs)):
            s.free(b, n)
        for turn in range(2):
            s.step([20, 9, 40, 17])                    # in blocks of this step
        s.free(2, 0)                                   # starts over; its blocks go to the others
        s.base[2] = 0
        s.step([60, 30, 21, 50])
        s.step([5, 0, 12, 1])
        # the rows of two sequences change places, with their lengths
        w.tables[:, [0, 3]] = w.tables[:, [3, 0]]
        s.base[[0, 3]] = s.base[[3, 0]]
        s.step([18, 33, 2, 7])
    finally:
        w.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_blocks_moved_between_a_step_and_its_commit(layout):
    s = Server(layout, False)
    w = s.w
    try:
        s.base = np.array([250, 16, 77, 100])

        def move():
            for l in range(w.L):
                for b in range(w.B):
                    for j in {s.base[b] // w.bs, (w.lens[b] - 1) // w.bs}:
                        s.migrate(l, b, j)
        for nodes in ([20, 9, 12, 17], [30, 3, 1, 40]):
            s.step(nodes, before_commit=move)
    finally:
        w.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_paths_as_long_as_the_trees(layout):
    """accept's own choice of a path's capacity: lists much shorter than it is."""
    s = Server(layout, False)
    w = s.w
    try:
        s.base = np.array([100, 5, 0, 33])
        kept = [s.step(nodes, cap=None) for nodes in ([16, 7, 12, 16], [3, 9, 0, 66], [64, 1, 40, 2])]
        assert max(k.max() for k in kept) > 2
    finally:
        w.close()


@pytest.mark.parametrize("checked", [False, True])
def test_steps_without_nodes_and_full_tables(checked):
    """No sequence has nodes; one has filled its table; one is empty; then all of a table is nodes."""
    s = Server(0, False, checked=checked)
    w = s.w
    try:
        full = w.tables.shape[2] * w.bs
        s.base = np.array([full, 0, 90, 170])
        assert s.step([0, 0, 0, 0], cap=None).tolist() == [0, 0, 0, 0]
        assert s.base.tolist() == [full, 0, 90, 170]
        s.base[0] = full - 33
        s.step([33, 1, 0, 5], cap=None)
        s.free(0, 0)
        s.base[0] = 0
        s.step([full, 0, 2, 1])
    finally:
        w.close()
