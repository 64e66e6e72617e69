"""The operators of include/ema_tree.h on the GPU against the oracle: masks and
positions of trees, attention of their nodes, the accepted path and the compaction;
odd sizes, empty requests, masks that leave rows empty, masked NaN, strides,
streams, graphs and invalid input."""
import numpy as np
import pytest
import torch

import oracle
import synth
from harness import TORCH_DT
from ops_harness import D, SmallCache, assert_close, dev16, i32, scores_bounded
from oracle import trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


@pytest.fixture(scope="module")
def small(ema):
    """A handle for calls that need no cache."""
    h = ema.slice_create(1, D, 16, "bf16", 0, 4 * 8192, 0)
    yield h
    ema.slice_destroy(h)


def i64(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int64)).cuda()


def full(shape, value=-99, dtype=torch.int32):
    return torch.full(shape, value, dtype=dtype, device="cuda")


def random_tree(rng, n, kind):
    i = np.arange(n)
    p = {"chain": i - 1, "star": np.minimum(i, 1) - 1, "roots": np.full(n, -1),
         "random": (rng.random(n) * (i + 1)).astype(int) - 1,
         "draft": np.maximum(np.where(rng.random(n) < 0.5, i - 1, i - 1 - rng.geometric(0.3, n)), 0)}[kind]
    if n:
        p[0] = -1
    return p


def forest(rng, sizes, kind):
    starts = np.concatenate([[0], np.cumsum(sizes)]).astype(int)
    parents = [random_tree(rng, n, kind) for n in sizes]
    return starts, np.concatenate(parents + [np.zeros(0, int)]).astype(int)


# ---- masks and positions -------------------------------------------------------------

@pytest.mark.parametrize("kind", ["chain", "star", "roots", "random", "draft"])
@pytest.mark.parametrize("sizes,words", [([1], 1), ([0], 1), ([5, 0, 1, 64, 63], 1), ([65, 3, 128, 0], 2),
                                         ([1, 300, 257], 5), ([1024, 1023, 7], 16), ([9], 16)])
def test_tables_match_the_oracle(ema, small, sizes, words, kind):
    rng = np.random.default_rng(len(sizes))
    starts, parents = forest(rng, sizes, kind)
    lens = np.array(sizes) + rng.integers(0, 5000, len(sizes))
    T = int(starts[-1])
    mask, pos, base = full((T + 2, words), -7, torch.int64), full((T + 2,)), full((len(sizes),))
    rows = np.concatenate([parents, [5, 9]])             # rows of no request: not looked at
    ema.tree_tables(small, i32(rows), i32(starts), i32(lens), mask, pos, base)
    want = trees.tree_tables(parents, starts, lens, words)
    assert np.array_equal(mask[:T].cpu().numpy().view(np.uint64), want[0])
    assert np.array_equal(pos[:T].cpu().numpy(), want[1])
    assert np.array_equal(base.cpu().numpy(), want[2])
    assert (mask[T:] == -7).all() and (pos[T:] == -99).all()
    alone = full((T + 2, words), -7, torch.int64)
    ema.tree_tables(small, i32(rows), i32(starts), i32(lens), alone)
    assert torch.equal(alone, mask)
    assert ema.slice_device_errors(small) == 0


def test_tables_count_what_is_out_of_range(ema, small):
    #          itself, below -1, fine  | past the word   | too short
    parents = [0, -5, 1] + [i - 1 for i in range(70)] + [-1, 0]
    starts, lens = [0, 3, 73, 75], [10, 100, 1]
    mask, pos, base = full((75, 1), -7, torch.int64), full((75,)), full((3,))
    ema.tree_tables(small, i32(parents), i32(starts), i32(lens), mask, pos, base)
    m = mask.cpu().numpy().view(np.uint64)[:, 0].tolist()
    assert m[:3] == [1, 2, 6] and pos[:3].cpu().tolist() == [7, 7, 8]
    assert m[3:67] == [(2 << i) - 1 for i in range(64)] and m[67:73] == [0] * 6
    assert pos[3:73].cpu().tolist() == [30 + i for i in range(64)] + [30] * 6
    assert m[73:] == [1, 3] and pos[73:].cpu().tolist() == [-1, 0]
    assert base.cpu().tolist() == [7, 30, -1]
    assert ema.slice_device_errors(small) == 2 + 1 + 1
    # starts that descend, pass the rows, do not begin at 0: clamped
    for starts, bad in (([0, 6, 2, 8], 1), ([0, 4, 6, 99], 1), ([2, 4, 6, 8], 1), ([-3, 4, 6, 8], 1),
                        ([0, 2 ** 31 - 1, -2 ** 31, 8], 3)):
        p = full((8,), -1)
        ema.tree_tables(small, p, i32(starts), i32([50, 50, 50]), full((8, 1), 0, torch.int64))
        assert ema.slice_device_errors(small) == bad, starts


# ---- accepted paths ------------------------------------------------------------------

@pytest.mark.parametrize("rooted", [True, False])
@pytest.mark.parametrize("kind", ["chain", "star", "roots", "random", "draft"])
@pytest.mark.parametrize("sizes,cap", [([1], 1), ([0, 1, 2], 3), ([7, 64, 65, 0, 130], 8),
                                       ([1024, 31], 2000), ([20] * 70, 5)])
def test_paths_match_the_oracle(ema, small, sizes, cap, kind, rooted):
    rng = np.random.default_rng(cap)
    starts, parents = forest(rng, sizes, kind)
    T, B = int(starts[-1]), len(sizes)
    vocab = 3                                            # many siblings alike
    drafted, choice = rng.integers(0, vocab, T), rng.integers(0, vocab, T)
    if kind == "chain":
        drafted[:], choice[:] = 1, 1                     # the longest path
    root = None if rooted else rng.integers(0, vocab, B)
    path, n, after = full((B, cap)), full((B,)), full((B,))
    ema.tree_accept(small, i32(parents), i32(starts), i32(drafted), i32(choice), path, n, after,
                    root_choice=None if rooted else i32(root))
    want = trees.tree_accept(parents, starts, drafted, choice, cap, root)
    for got, ref in zip((path, n, after), want):
        assert np.array_equal(got.cpu().numpy(), ref)
    assert ema.slice_device_errors(small) == 0


def test_paths_count_what_is_out_of_range(ema, small):
    # nodes 1 and 2 hang from nowhere; node 1024 is not looked at
    parents = np.concatenate([[-1, 1, -3, 0], np.arange(1025) - 1])
    starts = [0, 4, 1029]
    path, n, after = full((2, 1100)), full((2,)), full((2,))
    ones = full((1029,), 1)
    ema.tree_accept(small, i32(parents), i32(starts), ones, ones, path, n, after)
    assert path[0, :3].cpu().tolist() == [0, 3, -1] and n.cpu().tolist() == [2, 1024]
    assert path[1, :1025].cpu().tolist() == [*range(1024), -1] and after.cpu().tolist() == [1, 1]
    assert ema.slice_device_errors(small) == 2 + 1


# ---- attention -----------------------------------------------------------------------

class Case:
    """Requests of `lens` tokens whose last `new` are nodes with the given masks."""

    def __init__(self, ema, lens, new, heads, bs, dtype, seed=0, kind="draft", words=None, bits=None,
                 **kw):
        self.ema, self.c = ema, SmallCache(ema, lens, heads[1], bs, dtype, seed=seed, **kw)
        self.heads, self.dtype = heads, dtype
        self.starts, self.parents = forest(self.c.rng, new, kind)
        self.T = int(self.starts[-1])
        self.words = words or max(1, -(-max(new) // 64))
        base = [max(n, k) for n, k in zip(lens, new)]
        self.mask = trees.tree_tables(self.parents, self.starts, base, self.words)[0] \
            if bits is None else bits(self.c.rng, (self.T, self.words))
        self.q16 = self.c.queries(self.T, heads[0])

    def call(self, out, **kw):
        c = self.c
        self.ema.paged_tree_attention(c.h, kw.pop("q", dev16(self.q16, self.dtype)), i32(self.starts),
                                      kw.pop("table", c.table_dev), c.lens_dev, i64(self.mask), out,
                                      **kw)
        return out

    def out(self, dtype, rows=None):
        return full((self.T if rows is None else rows, self.heads[0], D), 7.0, dtype)

    def ref(self):
        c = self.c
        return trees.tree_attention(self.q16, self.starts, c.table, c.lens, self.mask, c.read_block,
                                    self.heads[1], D, c.bs, self.dtype)

    def check(self, got):
        want, mass = self.ref()
        assert_close(got, want, mass, got.dtype, self.dtype, int(self.c.lens.max()))

    def close(self):
        self.c.close()


SIZES = [
    # lens, new, (query heads, KV heads), block size, dtype
    ([1], [1], (2, 1), 16, "bf16"),
    ([17, 64, 65], [1, 1, 1], (4, 2), 16, "f16"),
    ([5, 0, 33, 130], [5, 0, 2, 7], (8, 2), 16, "bf16"),
    ([200, 64, 63, 1], [8, 8, 8, 1], (3, 3), 32, "f16"),
    ([100, 300, 77], [61, 64, 65], (6, 2), 64, "bf16"),           # row tiles of several nodes
    ([129, 700], [129, 200], (4, 1), 128, "f16"),
    ([1000, 31], [30, 31], (7, 1), 256, "bf16"),                  # a group that fills no tile
    ([515], [3], (16, 1), 16, "bf16"),
    ([90, 400], [33, 1], (17, 1), 16, "f16"),
    ([2100, 40, 900], [16, 16, 16], (8, 2), 16, "bf16"),
    ([70] * 40, [4] * 40, (4, 1), 16, "f16"),
    ([3000], [12], (32, 8), 16, "bf16"),
]


@pytest.mark.parametrize("full_weights", [False, True])
@pytest.mark.parametrize("out", ["f32", "same"])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_attention_matches_the_oracle(ema, case, out, full_weights):
    lens, new, heads, bs, dtype = SIZES[case]
    k = Case(ema, lens, new, heads, bs, dtype, seed=case, kind=["draft", "random", "roots"][case % 3])
    try:
        scores_bounded(k.c, k.q16)
        got = k.call(k.out(torch.float32 if out == "f32" else TORCH_DT[dtype]),
                     full_weights=full_weights)
        k.check(got)
        assert ema.slice_device_errors(k.c.h) == 0
    finally:
        k.close()


@pytest.mark.parametrize("heads,new", [((300, 1), [2, 1]), ((1030, 2), [1, 2]), ((64, 1), [40, 9])])
def test_large_groups(ema, heads, new):
    """Row tiles that begin and end inside a node's heads."""
    k = Case(ema, [70, 600], new, heads, 16, "bf16", seed=14)
    try:
        k.check(k.call(k.out(torch.float32)))
        k.check(k.call(k.out(torch.bfloat16)))
    finally:
        k.close()


@pytest.mark.parametrize("lens,new", [([40] * 700, [3] * 700), ([20000], [70]), ([9000, 3, 70, 1], [5, 3, 64, 1]),
                                      ([1500] * 70 + [1], [2] * 70 + [1])])
def test_many_requests_and_long_ones(ema, lens, new):
    """Whole items, equal shares of them, and a few in many parts; requests without nodes too."""
    k = Case(ema, lens, new, (4, 2), 16, "bf16", seed=15)
    try:
        k.check(k.call(k.out(torch.float32)))
        assert ema.slice_device_errors(k.c.h) == 0
    finally:
        k.close()


def test_an_empty_table_gives_zeros(ema):
    c = SmallCache(ema, [5], 2, 16, "bf16")
    try:
        o = torch.full((3, 4, D), 7.0, device="cuda")
        ema.paged_tree_attention(c.h, dev16(c.queries(3, 4), "bf16"), i32([0, 3]),
                                 torch.empty((1, 0), dtype=torch.int32, device="cuda"), i32([0]),
                                 full((3, 1), -1, torch.int64), o)
        assert (o == 0).all() and ema.slice_device_errors(c.h) == 1    # more nodes than tokens
    finally:
        c.close()


def test_a_16_bit_output_of_the_other_type(ema):
    k = Case(ema, [333, 20], [9, 20], (4, 2), 16, "f16", seed=3)
    try:
        k.check(k.call(k.out(torch.bfloat16)))
    finally:
        k.close()


@pytest.mark.parametrize("bs", [16, 32, 256])
@pytest.mark.parametrize("words", [1, 3])
def test_masks_of_any_bits(ema, words, bs):
    """Later nodes, not the row's own, none at all, and bits of no node."""
    def bits(rng, shape):
        m = rng.integers(0, 2 ** 63, shape, dtype=np.uint64) * np.uint64(2) + np.uint64(1)
        m[::5] = 0
        m[3::7] = ~np.uint64(0)
        return m
    k = Case(ema, [130, 71, 9, 65], [130, 70, 9, 1], (4, 2), bs, "bf16", seed=words, words=words,
             bits=bits)
    try:
        got = k.call(k.out(torch.float32))
        k.check(got)
        want, mass = k.ref()
        none = (mass == 0).all(axis=(1, 2))
        assert none.sum() >= 20 and (got.cpu().numpy()[none] == 0).all()
    finally:
        k.close()


def test_rows_of_no_request_stay_as_they_were(ema):
    k = Case(ema, [50, 40], [5, 6], (4, 2), 16, "bf16")
    try:
        k.mask = np.concatenate([k.mask, np.full((3, 1), 2 ** 64 - 1, np.uint64)])
        k.q16 = k.c.queries(14, 4)
        got = k.call(k.out(torch.bfloat16, rows=14))
        k.check(got)
        assert (got[11:] == 7).all()
    finally:
        k.close()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_values_that_are_not_finite_reach_who_attends_them(ema, out):
    inf, nan = 0x7F80, 0x7FC0
    k = Case(ema, [100, 40], [9, 6], (4, 2), 16, "bf16", seed=9, kind="star")
    try:
        c = k.c
        c.poke(1, 0, 91, 0, 5, inf)                      # the root of request 0
        c.poke(1, 0, 94, 1, 6, nan)                      # its node 3
        c.poke(0, 0, 96, 1, 0, nan)                      # K of its node 5
        c.poke(1, 1, 3, 0, 127, nan)                     # an older token of request 1
        c.poke(1, 1, 36, 1, 64, inf)                     # its node 2
        c.upload()
        got = k.call(k.out(out))
        finite = torch.isfinite(got).cpu().numpy()
        want = np.ones_like(finite)
        want[0:9, :2, 5] = False
        want[3, 2:, 6] = False
        want[5, 2:] = False
        want[9:15, :2, 127] = False
        want[11, 2:, 64] = False
        assert np.array_equal(finite, want)
        assert torch.isnan(got[5, 2:]).all() and torch.isnan(got[3, 2:, 6]).all()
        ref, mass = k.ref()
        ref[~want] = np.nan
        assert_close(torch.where(torch.from_numpy(want).cuda(), got, 0), np.where(want, ref, 0),
                     np.where(want, mass, 0), out, "bf16", 100)
    finally:
        k.close()


def test_infinite_keys(ema):
    """A score of -inf is no weight; one of +inf makes the row NaN."""
    k = Case(ema, [80, 33], [6, 4], (2, 1), 16, "bf16", seed=10, kind="roots")
    try:
        k.q16[:, :, 7] = 0x3F80                          # 1.0
        k.c.poke(0, 0, 12, 0, 7, 0xFF80)                 # an older token of request 0: -inf
        k.c.poke(0, 0, 76, 0, 7, 0xFF80)                 # its node 2, which attends itself
        k.c.poke(0, 1, 30, 0, 7, 0x7F80)                 # node 1 of request 1: +inf
        k.c.upload()
        got = k.call(k.out(torch.float32))
        with np.errstate(all="ignore"):
            want, mass = k.ref()
        assert np.isfinite(want[:6]).all() and torch.isnan(got[7]).all()
        keep = np.arange(10) != 7
        assert_close(got[torch.from_numpy(keep).cuda()], want[keep], mass[keep], torch.float32, "bf16", 80)
    finally:
        k.close()


def test_strided_queries(ema):
    k = Case(ema, [120, 77], [20, 7], (8, 2), 16, "bf16", seed=4)
    try:
        fused = torch.full((k.T, 8 + 4, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        fused[:, 2:10] = dev16(k.q16, "bf16")
        a = k.call(k.out(torch.bfloat16), q=fused[:, 2:10])
        b = k.call(k.out(torch.bfloat16))
        assert torch.equal(a, b)
        k.check(a)
    finally:
        k.close()


def test_a_scale(ema):
    k = Case(ema, [120, 77], [20, 7], (8, 2), 16, "f16", seed=5)
    try:
        got = k.call(k.out(torch.float32), scale=0.05)
        c = k.c
        want, mass = trees.tree_attention(k.q16, k.starts, c.table, c.lens, k.mask, c.read_block, 2, D,
                                          16, "f16", scale=0.05)
        assert_close(got, want, mass, torch.float32, "f16", 120)
    finally:
        k.close()


def test_the_table_s_width_and_the_blocks_places_do_not_matter(ema):
    a = Case(ema, [1700, 33, 400], [9, 9, 9], (8, 2), 16, "bf16", seed=6)
    try:
        one = a.call(a.out(torch.float32))
        wide = np.full((3, a.c.width + 900), -1)
        wide[:, :a.c.width] = a.c.table
        assert torch.equal(a.call(a.out(torch.float32), table=i32(wide)), one)
        assert ema.slice_device_errors(a.c.h) == 0
    finally:
        a.close()


@pytest.mark.parametrize("bs,lens,new", [(16, [16 * 90, 40], [33, 3]), (64, [700, 64], [5, 64]),
                                         (256, [600, 255], [100, 1])])
def test_bad_table_entries_are_left_out_and_counted_once(ema, bs, lens, new):
    """Block 0, full of NaN, must not be read in their place."""
    k = Case(ema, lens, new, (4, 2), bs, "bf16", seed=50)
    try:
        c = k.c
        spare = np.setdiff1d(np.arange(c.n_local), c.table)[0]
        c.local[[0, spare]] = c.local[[spare, 0]]
        c.table[c.table == 0] = spare
        c.upload()
        bad = c.table.copy()
        gone = [(0, 1), (1, 0)] + ([(0, 66), (0, 70)] if bs == 16 else [])
        for x, (b, j) in enumerate(gone):
            bad[b, j] = [-1, c.n_local, -2 ** 31, 2 ** 31 - 1][x]
        got = k.call(k.out(torch.float32), table=i32(bad)).cpu().numpy()
        assert np.isfinite(got).all() and ema.slice_device_errors(c.h) == len(gone)
        for b in (0, 1):                                 # as if the tokens there were not attended
            keep = [t for t in range(lens[b]) if (b, t // bs) not in gone]
            K, V = (oracle.to_float64(x, "bf16")[:, :] for x in
                    oracle.attention._gather_sequence(c.read_block, c.table[b], lens[b], 2, D, bs))
            base = lens[b] - new[b]
            for row in {k.starts[b], k.starts[b + 1] - 1}:
                sees = [t for t in keep if t < base or int(k.mask[row, (t - base) // 64]) >> ((t - base) % 64) & 1]
                q = oracle.to_float64(k.q16[row], "bf16")
                for h in range(4):
                    s = K[h // 2, sees] @ q[h] / np.sqrt(D)
                    w = np.exp(s - s.max(initial=0.0))
                    o = w @ V[h // 2, sees] / max(w.sum(), 1e-300)
                    assert np.abs(got[row, h] - o).max() < 1e-4
    finally:
        k.close()


def test_bad_starts_and_lengths_are_counted(ema):
    c = SmallCache(ema, [64, 40], 2, 16, "bf16", seed=53)
    try:
        q, mask = dev16(c.queries(10, 4), "bf16"), full((10, 1), -1, torch.int64)
        for starts, lens, bad in (([1, 3, 10], None, 1), ([0, 6, 2], None, 1), ([0, 12, 11], None, 2),
                                  ([-4, 3, 10], None, 1), ([0, 3, 2 ** 31 - 1], None, 1),
                                  ([0, 5, 10], [64, 2], 1), ([0, 5, 10], [-1, 40], 1),
                                  ([0, 5, 10], [2 ** 31 - 1, 40], 1)):
            o = torch.zeros((10, 4, D), device="cuda")
            ema.paged_tree_attention(c.h, q, i32(starts), c.table_dev,
                                     c.lens_dev if lens is None else i32(lens), mask, o)
            errors = ema.slice_device_errors(c.h)
            # (the longer length counts the table's unused entry too)
            assert errors == bad + (lens is not None and lens[0] > 64), (starts, lens)
    finally:
        c.close()


@pytest.mark.parametrize("B", [40, 2000])
def test_requests_of_the_same_rows(ema, B):
    """Starts that go up and down give every second request all rows: more items than the sizes
    allow for. They are counted, and the rows hold what one of them makes of them."""
    c = SmallCache(ema, [700, 600] * (B // 2), 2, 16, "bf16", seed=54) if B < 100 else \
        SmallCache(ema, [20] * B, 2, 16, "bf16", seed=54)
    try:
        q, mask = dev16(c.queries(60, 4), "bf16"), full((60, 1), -1, torch.int64)
        starts = np.zeros(B + 1, np.int64)
        starts[1::2] = 60
        o = torch.full((60, 4, D), 7.0, device="cuda")
        ema.paged_tree_attention(c.h, q, i32(starts), c.table_dev, c.lens_dev, mask, o)
        errors = ema.slice_device_errors(c.h)
        # the descending ones; where there are more rows than tokens, the others too
        assert errors == B // 2 + (0 if B < 100 else B // 2)
        assert torch.isfinite(o).all()
    finally:
        c.close()


def test_more_nodes_than_tokens(ema):
    """Rows at negative positions give zeros, the others attend the nodes that are there."""
    k = Case(ema, [40, 3], [6, 7], (4, 2), 16, "bf16", seed=11, kind="chain")
    try:
        got = k.call(k.out(torch.float32))
        assert (got[6:10] == 0).all()
        k.check(got)
        assert ema.slice_device_errors(k.c.h) == 1
    finally:
        k.close()


# ---- compaction ----------------------------------------------------------------------

class Pools:
    """Both pools with the requests' blocks scattered over them."""

    def __init__(self, ema, L, lens, heads, bs, layout, frac, seed=0, checked=False):
        self.ema, self.bs, self.H, self.nhd = ema, bs, heads, layout == 1
        rng = self.rng = np.random.default_rng(seed)
        nblk = -(-np.asarray(lens) // bs)
        N = L * int(nblk.sum())
        far = int(round(frac * N))
        self.n_local, self.n_far = N - far + 2, far + 1
        bb = 2 * bs * heads * D * 2
        self.h = ema.slice_create(heads, D, bs, "f16", layout, self.n_local * bb, self.n_far * bb,
                                  checked=checked)
        ids = np.concatenate([rng.permutation(self.n_local)[:N - far],
                              self.n_local + rng.permutation(self.n_far)[:far]])
        rng.shuffle(ids)
        self.table = np.full((L, len(lens), int(nblk.max(initial=0)) + 1), -1, np.int64)
        at = 0
        for l in range(L):
            for b, n in enumerate(nblk):
                self.table[l, b, :n] = ids[at:at + n]
                at += n
        self.views = [ema.pool_view(self.h, p) for p in (ema.POOL_LOCAL, ema.POOL_SLICE)]
        self.host = [rng.integers(0, 256, (n, bb), dtype=np.uint8) for n in (self.n_local, self.n_far)]
        for v, x in zip(self.views, self.host):
            v.copy_(torch.from_numpy(x))

    def expect(self, base, keep, n):
        return trees.kv_compact(*self.host, self.nhd, self.table, base, keep, n, self.H, D, self.bs)

    def same(self):
        torch.cuda.synchronize()
        for v, x in zip(self.views, self.host):
            assert np.array_equal(v.cpu().numpy(), x)

    def close(self):
        self.views = None
        torch.cuda.synchronize()
        self.ema.slice_destroy(self.h)


def lists(rng, base, lens, counts, extra=2):
    keep = np.full((len(base), max(counts) + extra), -5)
    for b, c in enumerate(counts):
        keep[b, :c] = np.sort(rng.permutation(lens[b] - base[b])[:c])
    return keep


COMPACT = [
    # layers, lens, bases, kept, KV heads, block size, part in the slice
    (1, [20], [3], [4], 1, 16, 0.0),
    (2, [40, 16, 0, 33], [10, 0, 0, 32], [5, 16, 0, 1], 2, 16, 0.5),
    (3, [100, 64, 129], [37, 0, 1], [17, 33, 100], 3, 32, 0.4),
    (2, [700, 256, 300], [0, 5, 255], [350, 1, 30], 2, 64, 1.0),
    (1, [1500], [0], [1200], 1, 128, 0.5),
    (2, [600, 500], [100, 0], [77, 499], 2, 256, 0.3),
    (5, [90] * 30, list(range(30)), [1 + i for i in range(30)], 8, 16, 0.3),
    (1, [2000, 1999], [1, 0], [1000, 40], 5, 16, 0.0),
]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("case", range(len(COMPACT)))
def test_compaction_matches_the_oracle(ema, case, layout):
    L, lens, base, counts, heads, bs, frac = COMPACT[case]
    p = Pools(ema, L, lens, heads, bs, layout, frac, seed=case)
    try:
        keep = lists(p.rng, base, lens, counts)
        new = full((len(lens),))
        ema.kv_compact(p.h, i32(p.table), i32(base), i32(keep), i32(counts), new_lens=new)
        want = p.expect(np.array(base), keep, counts)
        p.same()
        assert np.array_equal(new.cpu().numpy(), want)
        assert ema.slice_device_errors(p.h) == 0
    finally:
        p.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_empty_lists_and_tables(ema, layout):
    p = Pools(ema, 1, [20, 20], 1, 16, layout, 0.5)
    try:
        new = full((2,))
        none = torch.empty((2, 0), dtype=torch.int32, device="cuda")
        ema.kv_compact(p.h, i32(p.table), i32([3, 0]), none, i32([0, 0]), new_lens=new)
        assert new.cpu().tolist() == [3, 0]
        ema.kv_compact(p.h, none[None], i32([0, 0]), i32([[0, 1], [5, 6]]), i32([0, 2]), new_lens=new)
        assert new.cpu().tolist() == [0, 2] and ema.slice_device_errors(p.h) == 2
        p.same()
    finally:
        p.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_many_lists_long_and_short(ema, layout):
    """More requests than are put in order of their lists, and as many."""
    for B in (256, 300):
        rng = np.random.default_rng(B)
        lens = rng.integers(12, 130, B)
        p = Pools(ema, 1, lens, 1, 16, layout, 0.4, seed=B)
        try:
            base = rng.integers(0, 12, B)
            counts = [int(rng.integers(0, n - b + 1)) for n, b in zip(lens, base)]
            keep = lists(p.rng, base, lens, counts)
            ema.kv_compact(p.h, i32(p.table), i32(base), i32(keep), i32(counts))
            p.expect(base, keep, counts)
            p.same()
            assert ema.slice_device_errors(p.h) == 0
        finally:
            p.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_kept_heads_tails_and_all(ema, layout):
    """Nothing moves; all but the first; the first and last; windows behind some first ones."""
    for kept in (range(50), range(1, 50), [0, 49], [*range(4), *range(31, 50)], [49], []):
        p = Pools(ema, 2, [50 + 7], 2, 16, layout, 0.5, seed=len(kept))
        try:
            keep = np.array([list(kept) + [0]])
            ema.kv_compact(p.h, i32(p.table), i32([7]), i32(keep), i32([len(kept)]))
            p.expect(np.array([7]), keep, [len(kept)])
            p.same()
        finally:
            p.close()


def test_compaction_counts_what_is_out_of_range(ema):
    p = Pools(ema, 2, [48] * 6, 2, 16, 0, 0.5, seed=3)
    try:
        bad = p.table.copy()
        bad[1, 4, 1] = p.n_local + p.n_far               # layer 1: tokens 16..31 of request 4
        #        negative  fine  clamped  not ascending, past  bad block
        base = [-1, 0, 0, 20, 0, 0]
        n = [2, 2, 9, 4, 2, -3]
        keep = np.tile(np.array([1, 5, 6, 7]), (6, 1))
        keep[3] = [2, 1, 5, 60]
        keep[4] = [3, 20, 0, 0]
        new = full((6,))
        ema.kv_compact(p.h, i32(bad), i32(base), i32(keep), i32(n), new_lens=new)
        # (request, from, to) in order; request 3: entry 1 does not ascend, 3 is past the table
        moves = [(1, 1, 0), (1, 5, 1), (2, 1, 0), (2, 5, 1), (2, 6, 2), (2, 7, 3), (3, 22, 20),
                 (3, 25, 22), (4, 3, 0)]
        for l in range(2):
            for b, src, dst in moves + ([(4, 20, 1)] if l == 0 else []):
                trees.kv_compact(*p.host, False, p.table[l:l + 1, b:b + 1], [dst], [[src - dst]], [1],
                                 2, D, 16)
        p.same()
        assert new.cpu().tolist() == [1, 2, 4, 24, 2, 0]
        # negative base; 9 and -3; entries 1 and 3 of request 3; one token of one layer
        assert ema.slice_device_errors(p.h) == 1 + 2 + 2 + 1
    finally:
        p.close()


def test_a_checked_handle_refuses_on_the_host(ema):
    p = Pools(ema, 1, [40], 1, 16, 0, 0.0, checked=True)
    try:
        call = lambda keep, n: ema.kv_compact(p.h, i32(p.table), i32([0]), i32([keep]), i32([n]))
        call([1, 5], 2)
        for keep, n in (([5, 1], 2), ([1, 50], 2), ([1, 5], 3)):
            with pytest.raises(ema.EmaError):
                call(keep, n)
        with pytest.raises(ema.EmaError):
            ema.tree_tables(p.h, i32([1]), i32([0, 1]), i32([4]), full((1, 1), 0, torch.int64))
        with pytest.raises(ema.EmaError):
            ema.paged_tree_attention(p.h, torch.zeros((2, 1, D), dtype=torch.float16, device="cuda"),
                                     i32([0, 3]), i32(p.table[0]), i32([40]),
                                     full((2, 1), 0, torch.int64), torch.zeros((2, 1, D), device="cuda"))
        assert ema.slice_device_errors(p.h) == 0
    finally:
        p.close()


# ---- refusals of device arrays, streams, graphs ----------------------------------------

def test_refusals(ema):
    k = Case(ema, [40], [6], (4, 2), 16, "bf16")
    try:
        c, q, out = k.c, dev16(k.q16, "bf16"), k.out(torch.float32)
        starts, mask = i32(k.starts), i64(k.mask)
        ok = dict(q=q, query_start=starts, block_table=c.table_dev, seq_lens=c.lens_dev, mask=mask,
                  out=out)
        ema.paged_tree_attention(c.h, **ok)
        for bad in (dict(q=q.cpu()), dict(q=q.half()), dict(q=q[:, :3]), dict(mask=mask.int()),
                    dict(mask=mask[:5]), dict(mask=mask[:, 0]), dict(mask=mask.cpu()),
                    dict(mask=torch.cat([mask, mask], 1)[:, ::2]), dict(out=out[:5]),
                    dict(out=out.double()), dict(query_start=starts[:1]),
                    dict(query_start=starts.long()), dict(seq_lens=c.lens_dev[:0]),
                    dict(mask=torch.zeros((6, 17), dtype=torch.int64, device="cuda")),
                    dict(mask=torch.zeros((6, 0), dtype=torch.int64, device="cuda"))):
            with pytest.raises(ema.EmaError) as e:
                ema.paged_tree_attention(c.h, **{**ok, **bad})
            assert e.value.code == ema.ERR_INVAL
        need = ema.paged_tree_workspace(c.h, 6, 1, 4, c.width)
        if need:
            with pytest.raises(ema.EmaError):
                ema.paged_tree_attention(c.h, **ok, workspace=torch.empty(
                    need - 1, dtype=torch.uint8, device="cuda"))
        v = torch.empty(7, dtype=torch.int64, device="cuda").view(torch.int32)[1:13].view(6, 2)
        assert v.data_ptr() % 8 == 4
        p = full((6,), -1)
        rc = ema._lib.ema_tree_tables(c.h, p.data_ptr(), starts.data_ptr(), c.lens_dev.data_ptr(), 6,
                                      1, v.data_ptr(), 1, None, None, None)
        assert rc == ema.ERR_INVAL
        for bad in (dict(parents=p[:5]), dict(parents=p.cpu()), dict(seq_lens=c.lens_dev.long()),
                    dict(mask=mask.cpu()), dict(positions=p[:5]), dict(base=p)):
            with pytest.raises(ema.EmaError):
                ema.tree_tables(c.h, **{**dict(parents=p, query_start=starts, seq_lens=c.lens_dev,
                                               mask=mask), **bad})
    finally:
        k.close()


def step_calls(ema, k, T, words, st, bufs):
    """One tree step's calls over a case's cache, all on stream `st`."""
    c = k.c
    parents, starts, drafted, choice, q, mask, pos, base, out, path, n, after, lens, ws = bufs
    ema.tree_tables(c.h, parents, starts, c.lens_dev, mask, pos, base, stream=st)
    ema.paged_tree_attention(c.h, q, starts, c.table_dev, c.lens_dev, mask, out, workspace=ws, stream=st)
    ema.tree_accept(c.h, parents, starts, drafted, choice, path, n, after, stream=st)
    ema.kv_compact(c.h, c.table_dev[None], base, path, n, new_lens=lens, stream=st)


def step_buffers(ema, k):
    c, B = k.c, len(k.c.lens)
    drafted, choice = (c.rng.integers(0, 2, k.T) for _ in range(2))
    need = ema.paged_tree_workspace(c.h, k.T, B, k.heads[0], c.width)
    return (i32(k.parents), i32(k.starts), i32(drafted), i32(choice), dev16(k.q16, k.dtype),
            full((k.T, k.words), 0, torch.int64), full((k.T,)), full((B,)), k.out(torch.bfloat16),
            full((B, 6)), full((B,)), full((B,)), full((B,)),
            torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))


def test_a_step_in_a_graph_and_on_two_streams_at_once(ema):
    """Eager, replayed, and two requests' steps side by side on streams and in graphs."""
    ks = [Case(ema, [900, 45, 300], [16, 9, 40], (8, 2), 16, "bf16", seed=20 + i) for i in range(2)]
    try:
        bufs = [step_buffers(ema, k) for k in ks]
        first = [k.c.view.clone() for k in ks]
        want = []
        for k, b in zip(ks, bufs):
            step_calls(ema, k, k.T, k.words, None, b)
            torch.cuda.synchronize()
            k.check(b[8])
            want.append([x.clone() for x in b[5:13]] + [k.c.view.clone()])
        streams = [torch.cuda.Stream() for _ in ks]
        graphs = []
        for k, b, s in zip(ks, bufs, streams):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                step_calls(ema, k, k.T, k.words, s, b)
            graphs.append(g)
        for turn in range(4):
            for k, b, x in zip(ks, bufs, first):
                k.c.view.copy_(x)
                for t in b[5:13]:
                    t.fill_(-3)
            torch.cuda.synchronize()
            for k, b, s, g in zip(ks, bufs, streams, graphs):
                with torch.cuda.stream(s):
                    if turn % 2:
                        g.replay()
                    else:
                        step_calls(ema, k, k.T, k.words, s, b)
            torch.cuda.synchronize()
            for k, b, w in zip(ks, bufs, want):
                for got, ref in zip([*b[5:13], k.c.view], w):
                    assert torch.equal(got, ref)
            assert all(ema.slice_device_errors(k.c.h) == 0 for k in ks)
    finally:
        for k in ks:
            k.close()
