"""The operators of include/ema_ops.h on the GPU against float64: tables and
slot maps, the store of a chunk's tokens, attention of chunks and differential
attention; odd sizes, empty requests, masked NaN, strides, streams, graphs,
invalid input, and all of them together as a step uses them."""
import numpy as np
import pytest
import torch

import oracle
import synth
from harness import TORCH_DT
from ops_harness import D, SmallCache, assert_close, dev16, i32, scores_bounded
from oracle import ops as oops

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


# ---- tables ------------------------------------------------------------------------

def table_case(rng, L, lens, new, bs, slice_frac, slots, extra=1, room=2):
    """Random ids of both pools for the requests' blocks."""
    N = int((-(-np.asarray(lens) // bs)).sum())
    n_s = int(round(slice_frac * N))
    n_local = L * (N - n_s) + slots * n_s + 2
    n_slice = max(L * n_s, 1)
    loc, far = rng.permutation(n_local), rng.permutation(n_slice) + n_local
    ids = np.empty((L, N + extra), np.int64)
    for l in range(L):
        at = rng.permutation(N)
        ids[l, at[n_s:]] = loc[l * (N - n_s):(l + 1) * (N - n_s)]
        ids[l, at[:n_s]] = far[l * n_s:(l + 1) * n_s]
    ids[:, N:] = -7                                   # past every request: not looked at
    staging = loc[L * (N - n_s):][:slots * (n_s + 0)].reshape(slots, n_s) if n_s else None
    if staging is not None and room:
        staging = np.concatenate([staging, np.full((slots, room), 0)], axis=1)
    return ids, staging, n_local, n_slice


class TableOuts:
    """Device outputs full of a recognisable value."""

    def __init__(self, L, B, width, T, stage_n, cap, canon=True):
        f = lambda *s: torch.full(s, -99, dtype=torch.int32, device="cuda")
        self.table, self.slots, self.starts = f(L, B, width), f(L, T), f(B + 1)
        self.canon = f(L, B, width) if canon else None
        self.prefetch = (f(L, stage_n), f(L, stage_n), f(L))
        self.writeback = (f(L, cap), f(L, cap), f(L))


def run_tables(ema, h, ids, lens, new, o, staging, **kw):
    lists = {} if staging is None else dict(staging=i32(staging), prefetch=o.prefetch,
                                            writeback=o.writeback)
    ema.kv_tables(h, i32(ids), i32(lens), i32(new), o.table, o.slots, o.starts,
                  canon_table=o.canon, **lists, **kw)


def assert_tables(o, ref, staging):
    torch.cuda.synchronize()
    same = lambda t, r, what: np.testing.assert_array_equal(t.cpu().numpy(), r, what)
    same(o.starts, ref["starts"], "starts")
    same(o.table, ref["table"], "table")
    if o.canon is not None:
        same(o.canon, ref["canon"], "canon")
    same(o.slots, ref["slots"], "slots")
    if staging is not None:
        for kind in ("prefetch", "writeback"):
            for t, r, end in zip(getattr(o, kind), ref[kind], ("src", "dst", "n")):
                same(t, r, f"{kind} {end}")


@pytest.mark.parametrize("L,bs,frac,slots,seed,lens,new,width", [
    (1, 16, 0.0, 1, 0, [1], [1], 1),
    (1, 16, 0.0, 1, 1, [0], [0], 3),
    (2, 16, 1.0, 1, 2, [17], [17], 2),
    (3, 16, 0.5, 2, 3, [0, 1, 16, 17, 0, 33, 100, 0], [0, 1, 16, 2, 0, 0, 37, 0], 7),
    (2, 32, 0.3, 1, 4, [31, 32, 33, 64, 65], [31, 0, 33, 1, 64], 9),
    (5, 256, 0.4, 3, 5, [255, 256, 257, 1000], [1, 256, 3, 777], 4),
    # one block each: as many requests in a chunk as it has entries
    (2, 16, 0.5, 2, 6, [1 + i % 16 for i in range(5000)], [i % 2 for i in range(5000)], 1),
    # several chunks a layer, requests across their borders
    (3, 16, 0.4, 2, 7, [6000, 9001, 1, 0, 4095, 12007], [1, 9001, 1, 0, 100, 0], 751),
    (1, 16, 0.9, 1, 8, [900 + i for i in range(300)], [1 + i % 5 for i in range(300)], 77),
])
def test_tables_match_the_oracle(ema, L, bs, frac, slots, seed, lens, new, width):
    rng = np.random.default_rng(seed)
    ids, staging, n_local, n_slice = table_case(rng, L, lens, new, bs, frac, slots)
    bb = 2 * bs * D * 2
    h = ema.slice_create(1, D, bs, "bf16", 0, n_local * bb, n_slice * bb)
    try:
        T, cap = sum(new) + 3, 40 + sum(-(-n // bs) + 1 for n in new if n)
        stage_n = 0 if staging is None else staging.shape[1]
        o = TableOuts(L, len(lens), width, T, stage_n, cap, canon=seed != 4)
        run_tables(ema, h, ids, lens, new, o, staging)
        ref = oops.kv_tables(ids, lens, new, width, bs, n_local, T, staging, cap)
        assert_tables(o, ref, staging)
        assert ema.slice_device_errors(h) == 0
    finally:
        ema.slice_destroy(h)


def test_tables_of_no_requests(ema):
    h = ema.slice_create(1, D, 16, "bf16", 0, 4 * 8192, 8192)
    try:
        o = TableOuts(2, 0, 3, 5, 0, 1)
        run_tables(ema, h, np.zeros((2, 1)), [], [], o, None)
        torch.cuda.synchronize()
        assert (o.slots == -1).all() and o.starts.item() == 0
    finally:
        ema.slice_destroy(h)


def test_tables_count_and_clamp_what_is_out_of_range(ema):
    bb = 2 * 16 * D * 2
    h = ema.slice_create(1, D, 16, "bf16", 0, 10 * bb, 4 * bb)
    try:
        staging = np.array([[8]])                                # room for one slice block
        #        too long      more new than tokens   bad id, two slice blocks
        lens, new = [200, 3, 64], [0, 9, 20]
        ids = np.array([[0, 1, 2, 3, 99, 10, 11, 4]])
        o = TableOuts(1, 3, 3, 30, 1, 1)
        run_tables(ema, h, ids, lens, new, o, staging)
        torch.cuda.synchronize()
        assert o.table.cpu().numpy()[0].tolist() == [[0, 1, 2], [3, -1, -1], [-1, 8, -1]]
        assert o.canon.cpu().numpy()[0].tolist() == [[0, 1, 2], [3, -1, -1], [-1, 10, 11]]
        assert o.starts.cpu().tolist() == [0, 0, 3, 23]
        # the third request is cut to 48 tokens, new ones from 28 on: row 12 of block 8
        want = [48, 49, 50] + [8 * 16 + 12 + i for i in range(4)] + [-1] * 23
        assert o.slots.cpu().tolist()[0] == want
        # lengths 200, 64 and new 9; id 99; the second slice block and the write-back of it;
        # 16 new tokens in that block
        assert ema.slice_device_errors(h) == 3 + 1 + 2 + 16
        # fewer ids and slots than needed: the rest is left out
        o = TableOuts(1, 1, 3, 2, 1, 1)
        run_tables(ema, h, np.array([[5, 6]]), [40], [4], o, staging)
        torch.cuda.synchronize()
        assert o.table.cpu().tolist() == [[[5, 6, -1]]] and o.slots.cpu().tolist() == [[-1, -1]]
        assert ema.slice_device_errors(h) == 1 + 4
    finally:
        ema.slice_destroy(h)


# ---- store -----------------------------------------------------------------------------

def slots_of(table, lens, new, bs):
    out = []
    for b, (n, m) in enumerate(zip(lens, new)):
        out += [table[b, p // bs] * bs + p % bs for p in range(n - m, n)]
    return np.array(out, np.int64)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bs,H,lens,new", [
    (16, 2, [1], [1]),
    (16, 1, [7, 8, 9, 16, 17], [7, 8, 1, 16, 17]),
    (16, 8, [33, 100, 64, 5], [20, 73, 64, 1]),
    (32, 2, [200], [197]),
    (64, 3, [65, 130], [63, 100]),
    (128, 1, [129, 300], [129, 7]),
    (256, 2, [511, 3], [200, 3]),
])
def test_store_matches_the_oracle_bit_for_bit(ema, bs, H, lens, new, dtype):
    c = SmallCache(ema, lens, H, bs, dtype, seed=len(lens) + bs)
    try:
        slots = slots_of(c.table, lens, new, bs)
        T = len(slots)
        drop = c.rng.random(T) < 0.1
        slots[drop] = -1
        k, v = (synth.random_16bit(c.rng, (T, H, D), dtype) for _ in range(2))
        if bs == 16:                                  # rows of a fused projection
            qkv = synth.random_16bit(c.rng, (T, 3 + 2 * H, D), dtype)
            qkv[:, 3:3 + H], qkv[:, 3 + H:] = k, v
            q = dev16(qkv, dtype)
            kd, vd = q[:, 3:3 + H], q[:, 3 + H:]
        else:
            kd, vd = dev16(k, dtype), dev16(v, dtype)
        ema.kv_store(c.h, kd, vd, i32(slots))
        oops.kv_store(c.local, k, v, slots, H, D, bs)
        torch.cuda.synchronize()
        assert np.array_equal(c.view.cpu().numpy(), c.local)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()


def test_store_of_scattered_slots_and_a_slot_past_the_pool(ema):
    c = SmallCache(ema, [160] * 4, 2, 16, "bf16", seed=9)
    try:
        T = 150
        slots = c.rng.permutation(c.n_local * 16)[:T]
        slots[3:19] = np.arange(16) + 32                 # two groups off the tile's start
        slots[60:76] = np.arange(16) + 64                # a group across a tile's end
        used, first = np.unique(slots, return_index=True)
        slots[np.setdiff1d(np.arange(T), first)] = -1
        k, v = (synth.random_16bit(c.rng, (T, 2, D), "bf16") for _ in range(2))
        oops.kv_store(c.local, k, v, slots, 2, D, 16)
        bad = slots.copy()
        at = np.nonzero(slots == -1)[0]
        far = [c.n_local * 16, 2 ** 31 - 1, -2][:len(at)]
        bad[at[:len(far)]] = far
        ema.kv_store(c.h, dev16(k, "bf16"), dev16(v, "bf16"), i32(bad))
        torch.cuda.synchronize()
        assert np.array_equal(c.view.cpu().numpy(), c.local)
        assert ema.slice_device_errors(c.h) == len(far)
    finally:
        c.close()


# ---- attention ---------------------------------------------------------------------------

OUTS = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def run_attention(ema, c, q16, starts, out_dtype, maps, lam=None, norm=None, pad=0, scale=0.0,
                  strided=False, single=False, **kw):
    """The operator's output, with `pad` rows behind the last request."""
    T, Hq = q16.shape[:2]
    if strided:
        wide = np.zeros((T, Hq + 5, D), np.uint16)
        wide[:, 2:2 + Hq] = q16
        q = dev16(wide, c.dtype)[:, 2:2 + Hq]
    else:
        q = dev16(q16, c.dtype)
    out = torch.full((T, Hq // maps, maps * D), 7.0, dtype=out_dtype, device="cuda")
    if maps == 1:
        ema.paged_prompt_attention(c.h, q, i32(starts), c.table_dev, c.lens_dev, out, scale=scale,
                                   **kw)
        return out
    more = dict(norm_weight=None if norm is None else torch.tensor(norm, device="cuda"),
                norm_eps=1e-5, scale=scale, **kw)
    lam = torch.tensor(lam, device="cuda")
    if single:
        ema.paged_diff_attention(c.h, q, c.table_dev, c.lens_dev, lam, out, **more)
    else:
        ema.paged_diff_prompt_attention(c.h, q, i32(starts), c.table_dev, c.lens_dev, lam, out,
                                        **more)
    return out


def check_attention(ema, c, new, Hq, out, maps, norm=False, pad=0, scale=0.0, strided=False,
                    single=False):
    starts = np.concatenate([[0], np.cumsum(new)])
    q16 = c.queries(int(starts[-1]) + pad, Hq)
    scores_bounded(c, q16)
    rng = np.random.default_rng(Hq)
    lam = (rng.random(Hq // 2) + 0.1).astype(np.float32) if maps == 2 else None
    w = (rng.random(2 * D) + 0.5).astype(np.float32) if norm else None
    got = run_attention(ema, c, q16, starts, OUTS[out], maps, lam, w, scale=scale, strided=strided,
                        single=single)
    torch.cuda.synchronize()
    ref, mass = oops.prompt_attention(q16, starts, c.table, c.lens, c.read_block, c.H, D, c.bs,
                                      c.dtype, scale=scale if scale > 0 else None, lam=lam,
                                      norm_weight=w, norm_eps=1e-5)
    assert_close(got, ref, mass, OUTS[out], c.dtype, int(c.lens.max()), norm)
    if pad:
        assert (got[int(starts[-1]):] == 7.0).all()
    return got, ref


PROMPTS = [
    # lens, new, kv heads, query heads, block size
    ([1], [1], 1, 1, 16),
    ([5, 0, 17], [5, 0, 16], 2, 2, 16),
    ([40, 16, 33, 1], [40, 1, 0, 1], 1, 4, 16),
    ([129, 64, 65], [129, 63, 65], 2, 6, 16),            # three query heads per KV head
    ([300, 31], [260, 31], 1, 8, 32),
    ([500, 64], [3, 64], 2, 16, 64),
    ([257, 130], [128, 129], 1, 3, 128),
    ([700], [90], 1, 16, 256),
    ([2100, 1025], [2, 1], 2, 4, 16),                    # few rows, long axis
]


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"),
                                       ("f16", "f32")])
@pytest.mark.parametrize("lens,new,H,Hq,bs", PROMPTS)
def test_prompt_attention(ema, lens, new, H, Hq, bs, dtype, out):
    c = SmallCache(ema, lens, H, bs, dtype, seed=sum(lens))
    try:
        check_attention(ema, c, new, Hq, out, 1, pad=3, strided=Hq == 8)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()


@pytest.mark.parametrize("dtype,out,norm", [("bf16", "bf16", True), ("f16", "f16", False),
                                            ("bf16", "f32", True), ("f16", "f32", False)])
@pytest.mark.parametrize("lens,new,H,Hq,bs", [(l, n, 2 * H, 2 * Hq, bs)
                                              for l, n, H, Hq, bs in PROMPTS])
def test_diff_prompt_attention(ema, lens, new, H, Hq, bs, dtype, out, norm):
    c = SmallCache(ema, lens, H, bs, dtype, seed=sum(lens) + 1)
    try:
        check_attention(ema, c, new, Hq, out, 2, norm=norm, pad=2, strided=Hq == 16)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()


@pytest.mark.parametrize("dtype,out,norm", [("bf16", "bf16", True), ("f16", "f32", False),
                                            ("bf16", "f32", True), ("f16", "f16", False)])
@pytest.mark.parametrize("lens,H,Hq,bs", [
    ([1], 2, 2, 16),
    ([0, 5, 0], 2, 4, 16),
    ([16, 17, 31, 32, 33, 64, 65], 4, 4, 16),
    ([100, 900, 1, 333], 2, 16, 32),
    ([1500, 20], 2, 6, 64),
    ([4097], 4, 16, 128),
    ([600, 257, 255], 2, 4, 256),
    (list(range(1, 400, 7)), 2, 8, 16),
    ([130, 77], 2, 32, 16),                              # 16 query heads per KV head
])
def test_diff_attention(ema, lens, H, Hq, bs, dtype, out, norm):
    c = SmallCache(ema, lens, H, bs, dtype, seed=sum(lens) + 2)
    try:
        check_attention(ema, c, [1] * len(lens), Hq, out, 2, norm=norm, strided=Hq == 16,
                        single=True)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()


@pytest.mark.parametrize("single", [True, False])
def test_a_zero_row_stays_zero_under_the_norm(ema, single):
    """One token and lambda 1: both maps are 1, their difference 0, and without an
    epsilon its norm is 0 / 0."""
    c = SmallCache(ema, [1, 1, 0], 2, 16, "bf16", seed=25)
    try:
        B = len(c.lens)
        q = dev16(c.queries(B, 4), "bf16")
        lam, w = torch.ones(2, device="cuda"), torch.full((256,), 3.0, device="cuda")
        out = torch.full((B, 2, 256), 7.0, device="cuda")
        if single:
            ema.paged_diff_attention(c.h, q, c.table_dev, c.lens_dev, lam, out, norm_weight=w)
        else:
            ema.paged_diff_prompt_attention(c.h, q[:2], i32([0, 1, 2, 2]), c.table_dev, c.lens_dev,
                                            lam, out[:2], norm_weight=w)
            assert torch.all(out[2] == 7.0)
            out = out[:2]
        assert torch.all(out == 0)
    finally:
        c.close()


@pytest.mark.parametrize("maps", [1, 2])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f32")])
def test_many_query_heads_per_kv_head(ema, maps, dtype, out):
    c = SmallCache(ema, [130, 40], 2, 16, dtype, seed=26)
    try:
        check_attention(ema, c, [21, 40], 80, out, maps)
    finally:
        c.close()


@pytest.mark.parametrize("maps", [1, 2])
def test_scale_and_output_of_the_other_type(ema, maps):
    c = SmallCache(ema, [70, 40], 2, 16, "f16", seed=20)
    try:
        check_attention(ema, c, [33, 40], 4, "bf16", maps, scale=0.21)
    finally:
        c.close()


@pytest.mark.parametrize("maps", [1, 2])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_masked_tokens_may_hold_anything(ema, maps, dtype):
    """Infinities and NaN in later tokens of the chunk reach only the rows that
    attend them (as something not finite), in the channels that hold them."""
    inf = {"bf16": 0x7F80, "f16": 0x7C00}[dtype]
    n, new, H = 90, 70, 2
    clean = SmallCache(ema, [n, 40], H, 16, dtype, seed=21)
    c = SmallCache(ema, [n, 40], H, 16, dtype, seed=21)
    try:
        c.poke(1, 0, 75, 0, 5, synth.NAN16[dtype])
        c.poke(1, 0, 80, 0, 6, inf)
        c.poke(1, 0, 81, 1, 7, inf | 0x8000)
        c.poke(0, 0, 85, 0, 9, synth.NAN16[dtype])
        c.poke(0, 0, 85, 1, 9, synth.NAN16[dtype])
        c.upload()
        q16 = c.queries(new + 40, 4)
        starts = [0, new, new + 40]
        lam = np.array([0.5, 0.25], np.float32)
        a, b = (run_attention(ema, x, q16, starts, torch.float32, maps, lam).cpu().numpy()
                for x in (clean, c))
        at = lambda t: t - (n - new)                      # row of position t
        a, b = (x.reshape(new + 40, 2, 2 * D) for x in (a, b))
        # what every kernel has to keep: rows before a token, and the other request
        assert np.array_equal(a[:at(75)], b[:at(75)]) and np.array_equal(a[new:], b[new:])
        assert np.isnan(b[at(85):new]).all()              # their scores are NaN
        mid = b[at(75):at(85)]
        touched = np.zeros(2 * D, bool)
        touched[[5, 6, 7, D + 5, D + 6, D + 7]] = True
        assert np.isfinite(mid[..., ~touched]).all()
        assert np.isnan(mid[:, 0, 5]).all()
        assert not np.isfinite(b[at(80):at(85), 0, 6]).any()
        assert np.isfinite(b[:at(80), 0, 6]).all()
    finally:
        c.close()
        clean.close()


def test_bad_table_entries_are_masked_and_counted(ema):
    c = SmallCache(ema, [64, 40], 2, 16, "bf16", seed=22)
    try:
        q16 = c.queries(10, 4)
        starts = [0, 4, 10]
        table = c.table.copy()
        table[0, 1] = c.n_local                            # tokens 16..31 of request 0
        table[1, 0] = -1
        c.table_dev = i32(table)
        lam = np.array([0.5, 0.25], np.float32)
        for maps in (1, 2):
            got = run_attention(ema, c, q16, starts, torch.float32, maps, lam)
            assert ema.slice_device_errors(c.h) > 0
            # the same with those tokens left out of a cache of their own
            from oracle.attention import _gather_sequence
            for b, (r0, r1, gone) in enumerate(((0, 4, (16, 32)), (4, 10, (0, 16)))):
                n = int(c.lens[b])
                K, V = _gather_sequence(c.read_block, c.table[b], n, 2, D, 16)
                K, V = (oracle.to_float64(x, "bf16") for x in (K, V))
                for row in range(r0, r1):
                    seen = n - (r1 - row) + 1
                    keep = [t for t in range(seen) if not gone[0] <= t < gone[1]]
                    q = oracle.to_float64(q16[row], "bf16")
                    w = [oops._weights(q[h], K[h // 2 if maps == 1 else h % 2, keep], D ** -0.5)
                         for h in range(4)]
                    if maps == 1:
                        ref = np.stack([w[h] @ V[h // 2, keep] for h in range(4)])
                    else:
                        v = np.concatenate([V[0, keep], V[1, keep]], axis=1)
                        ref = np.stack([(w[2 * h] - lam[h] * w[2 * h + 1]) @ v for h in range(2)])
                    assert np.abs(got[row].double().cpu().numpy() - ref).max() < 1e-4
    finally:
        c.close()


def test_more_queries_than_tokens_give_zeros(ema):
    c = SmallCache(ema, [3, 20], 2, 16, "bf16", seed=23)
    try:
        q16 = c.queries(25, 2)
        for maps, lam in ((1, None), (2, np.array([0.5], np.float32))):
            got = run_attention(ema, c, q16, [0, 5, 25], torch.float32, maps, lam)
            torch.cuda.synchronize()
            assert (got[:2] == 0).all() and (got[2:] != 0).any(dim=-1).all()
            assert ema.slice_device_errors(c.h) > 0
    finally:
        c.close()


# ---- streams and graphs -------------------------------------------------------------------

def test_two_streams_at_once_and_graph_replays(ema):
    """Calls on one handle on two streams, and two captured graphs replayed at once,
    each against the eager result, several times."""
    c = SmallCache(ema, [1200, 900, 40], 2, 16, "bf16", seed=24)
    try:
        starts = i32([0, 2, 34, 40])
        qs = [dev16(c.queries(40, 4), "bf16") for _ in range(2)]
        lam = torch.tensor([0.5, 0.3], device="cuda")
        single = [q[:3].contiguous() for q in qs]

        def calls(i, outs, stream=None):
            ema.paged_prompt_attention(c.h, qs[i], starts, c.table_dev, c.lens_dev, outs[0],
                                       stream=stream)
            ema.paged_diff_prompt_attention(c.h, qs[i], starts, c.table_dev, c.lens_dev, lam,
                                            outs[1], stream=stream)
            ema.paged_diff_attention(c.h, single[i], c.table_dev, c.lens_dev, lam, outs[2],
                                     stream=stream)

        new_outs = lambda: [torch.zeros((40, 4, D), dtype=torch.bfloat16, device="cuda"),
                            torch.zeros((40, 2, 2 * D), dtype=torch.bfloat16, device="cuda"),
                            torch.zeros((3, 2, 2 * D), dtype=torch.bfloat16, device="cuda")]
        want = [new_outs() for _ in range(2)]
        for i in (0, 1):
            calls(i, want[i])
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = [new_outs() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(10):
            for i in (0, 1):
                calls(i, got[i], streams[i])
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(want[i], got[i]))
        graphs = []
        for i in (0, 1):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=streams[i]):
                calls(i, got[i])
            graphs.append(g)
        for _ in range(4):
            for o in got[0] + got[1]:
                o.zero_()
            calls(0, new_outs())                           # eager work between the replays
            torch.cuda.synchronize()
            for i in (0, 1):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay()
            torch.cuda.synchronize()
            for i in (0, 1):
                assert all(torch.equal(a, b) for a, b in zip(want[i], got[i]))
        del graphs
    finally:
        c.close()


def test_own_workspace_and_one_too_small(ema):
    c = SmallCache(ema, [5000], 2, 16, "bf16", seed=25)
    try:
        q = dev16(c.queries(2, 2), "bf16")
        out = torch.empty((2, 2, D), dtype=torch.bfloat16, device="cuda")
        ref = torch.empty_like(out)
        n = ema.paged_prompt_workspace(c.h, 2, 1, 2, c.width)
        ema.paged_prompt_attention(c.h, q, i32([0, 2]), c.table_dev, c.lens_dev, ref)
        ws = torch.full((n + 16,), 255, dtype=torch.uint8, device="cuda")   # NaN all over
        ema.paged_prompt_attention(c.h, q, i32([0, 2]), c.table_dev, c.lens_dev, out,
                                   workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
        if n:
            with pytest.raises(ema.EmaError):
                ema.paged_prompt_attention(c.h, q, i32([0, 2]), c.table_dev, c.lens_dev, out,
                                           workspace=ws[:n - 1])
    finally:
        c.close()


# ---- refusals on the device path ---------------------------------------------------------

def test_arguments_that_are_refused(ema):
    c = SmallCache(ema, [20], 2, 16, "bf16", seed=26)
    try:
        q = dev16(c.queries(4, 2), "bf16")
        out = torch.empty((4, 2, D), dtype=torch.bfloat16, device="cuda")
        ok = (q, i32([0, 4]), c.table_dev, c.lens_dev, out)
        lam = torch.ones(1, device="cuda")
        slots = i32([0, 1, 2, 3])
        kv = q[:, :2]

        def refused(fn, *a, **kw):
            with pytest.raises(ema.EmaError) as e:
                fn(c.h, *a, **kw)
            assert e.value.code == ema.ERR_INVAL

        f = ema.paged_prompt_attention
        f(c.h, *ok)
        refused(f, q.half(), *ok[1:])                              # another type
        refused(f, q.cpu(), *ok[1:])
        refused(f, q.transpose(0, 1), *ok[1:])                     # heads apart
        refused(f, q, i32([0]), *ok[2:])                           # starts too short
        refused(f, q, ok[1].long(), *ok[2:])
        refused(f, *ok[:4], out[:3])                               # out too small
        refused(f, *ok[:4], out.double())
        refused(f, dev16(c.queries(4, 3), "bf16"), *ok[1:])        # 3 query, 2 KV heads
        wide = torch.zeros((4, 2 * D + 4), dtype=torch.bfloat16, device="cuda")
        refused(f, wide[:, :2 * D].unflatten(1, (2, D)), *ok[1:])  # stride 260
        refused(f, wide.view(-1)[4:4 + 4 * 2 * D].view(4, 2, D), *ok[1:])   # not 16-byte aligned
        refused(ema.paged_diff_prompt_attention, *ok[:4], lam.half(), out.view(4, 1, 256))
        refused(ema.paged_diff_prompt_attention, *ok[:4], lam, out.view(4, 1, 256),
                norm_weight=torch.ones(255, device="cuda"))
        refused(ema.paged_diff_prompt_attention, *ok[:4], lam, out.view(4, 1, 256), norm_eps=-1.0)
        refused(ema.paged_diff_attention, q, c.table_dev, c.lens_dev, lam, out)   # 4 rows, 1 request
        refused(ema.kv_store, kv, kv[:3], slots)
        refused(ema.kv_store, kv, kv, slots[:3])
        refused(ema.kv_store, kv[:, :1], kv[:, :1], slots)
        refused(ema.kv_store, kv.float(), kv.float(), slots)
        torch.cuda.synchronize()
    finally:
        c.close()


def test_checked_handles_read_the_arrays_back(ema):
    c = SmallCache(ema, [20, 33], 2, 16, "bf16", seed=27, checked=True)
    try:
        q = dev16(c.queries(6, 2), "bf16")
        out = torch.empty((6, 2, D), dtype=torch.bfloat16, device="cuda")
        call = lambda starts, table, lens: ema.paged_prompt_attention(
            c.h, q, i32(starts), i32(table), i32(lens), out)
        call([0, 2, 6], c.table, c.lens)
        bad = c.table.copy()
        bad[1, 2] = c.n_local
        for a in (([0, 2, 7], c.table, c.lens), ([1, 2, 6], c.table, c.lens),
                  ([0, 4, 3], c.table, c.lens), ([0, 2, 6], bad, c.lens),
                  ([0, 2, 6], c.table, [20, 65]), ([0, 2, 6], c.table, [1, 33])):
            with pytest.raises(ema.EmaError):
                call(*a)
        with pytest.raises(ema.EmaError):
            ema.kv_store(c.h, q, q, i32([0, 1, 2, 3, 4, 0]))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            with pytest.raises(ema.EmaError):
                ema.paged_prompt_attention(c.h, q, c.lens_dev, c.table_dev, c.lens_dev, out)
            out.zero_()
        del g
    finally:
        c.close()


# ---- larger grids, batches and pools -------------------------------------------------------

def test_tables_large_enough_for_the_larger_chunks(ema):
    L, B, width, bs = 3, 1000, 720, 16
    rng = np.random.default_rng(40)
    lens = rng.integers(0, 700, B)
    lens[[0, 500, 999]] = [width * bs, 0, width * bs - 5]
    new = np.minimum(lens, rng.integers(0, 40, B))
    new[0] = 3000
    ids, staging, n_local, n_slice = table_case(rng, L, lens, new, bs, 0.4, 2)
    bb = 2 * bs * D * 2
    h = ema.slice_create(1, D, bs, "bf16", 0, n_local * bb, n_slice * bb)
    try:
        T, cap = int(new.sum()), int((-(-new // bs) + 1).sum())
        o = TableOuts(L, B, width, T, staging.shape[1], cap)
        run_tables(ema, h, ids, lens, new, o, staging)
        assert_tables(o, oops.kv_tables(ids, lens, new, width, bs, n_local, T, staging, cap),
                      staging)
        assert ema.slice_device_errors(h) == 0
    finally:
        ema.slice_destroy(h)


@pytest.mark.parametrize("maps,out", [(1, "bf16"), (1, "f32"), (2, "bf16"), (2, "f32")])
def test_more_sequences_than_a_wave_searches(ema, maps, out):
    rng = np.random.default_rng(41)
    lens = rng.integers(0, 40, 700)
    lens[[3, 699]] = [400, 333]
    new = np.minimum(lens, rng.integers(0, 6, 700))
    new[[3, 699]] = [150, 40]
    c = SmallCache(ema, lens, 2, 16, "bf16", seed=41, extra_width=0)
    try:
        check_attention(ema, c, new.tolist(), 4, out, maps, pad=1)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()


def test_differential_decode_of_more_pairs_than_workgroups(ema):
    rng = np.random.default_rng(42)
    lens = rng.integers(0, 300, 350)
    lens[[0, 7, 200, 349]] = [3000, 0, 1700, 33]
    c = SmallCache(ema, lens, 2, 16, "f16", seed=42)
    try:
        check_attention(ema, c, [1] * 350, 4, "f32", 2, single=True)
        check_attention(ema, c, [1] * 350, 2, "f16", 2, norm=True, single=True)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()


def test_blocks_past_four_gibibytes(ema):
    """A pool of 5 GiB whose last blocks are used: offsets take more than 32 bits."""
    H, bs, n = 8, 256, 5120                              # blocks of 1 MiB
    bb = 2 * bs * H * D * 2
    small = SmallCache(ema, [600, 300], H, bs, "bf16", seed=43, spare=0)
    h = ema.slice_create(H, D, bs, "bf16", 0, n * bb, 0)
    try:
        view = ema.pool_view(h, ema.POOL_LOCAL)
        first = n - small.n_local
        view[first:].copy_(small.view)
        table = i32(np.where(small.table >= 0, small.table + first, -1))
        q = dev16(small.queries(40, 16), "bf16")
        k, v = (dev16(small.queries(3, H), "bf16") for _ in range(2))
        slots = np.array([5, 70, 511]) + (small.table[1, 0] * bs)
        lam = torch.linspace(0.1, 0.9, 8, device="cuda")
        starts, one = i32([0, 30, 40]), q[:2].contiguous()
        got = []
        for hh, t, s in ((small.h, small.table_dev, slots), (h, table, slots + first * bs)):
            ok = i32(np.where(slots // bs == small.table[1, 0], s, -1))
            ema.kv_store(hh, k, v, ok)
            outs = [torch.zeros((40, 16, D), dtype=torch.bfloat16, device="cuda"),
                    torch.zeros((40, 8, 2 * D), dtype=torch.bfloat16, device="cuda"),
                    torch.zeros((2, 8, 2 * D), dtype=torch.bfloat16, device="cuda")]
            ema.paged_prompt_attention(hh, q, starts, t, small.lens_dev, outs[0])
            ema.paged_diff_prompt_attention(hh, q, starts, t, small.lens_dev, lam, outs[1])
            ema.paged_diff_attention(hh, one, t, small.lens_dev, lam, outs[2])
            torch.cuda.synchronize()
            got.append(outs)
        assert all(torch.equal(a, b) for a, b in zip(*got))
        assert torch.equal(view[first:], small.view)
        view = None
    finally:
        view = None
        small.close()
        ema.slice_destroy(h)


def test_results_do_not_depend_on_placement_or_width(ema):
    """The same tokens in other blocks and a wider table: the same bits (the width decides how
    the work is cut only where rows are few)."""
    a = SmallCache(ema, [700, 90], 2, 16, "bf16", seed=44)
    b = SmallCache(ema, [700, 90], 2, 16, "bf16", seed=44, spare=3)
    try:
        perm = np.random.default_rng(1).permutation(a.n_local)
        b.local[perm] = a.local
        b.upload()
        b.table_dev = i32(np.where(a.table >= 0, perm[a.table], -1))
        q16 = a.queries(400, 4)
        starts = [0, 350, 400]
        lam = np.array([0.5, 0.25], np.float32)
        for maps in (1, 2):
            x, y = (run_attention(ema, c, q16, starts, torch.float32, maps, lam) for c in (a, b))
            torch.cuda.synchronize()
            assert torch.equal(x, y)
    finally:
        a.close()
        b.close()


@pytest.mark.parametrize("maps", [1, 2])
def test_a_workspace_of_another_stream_is_no_memory_still_in_use(ema, maps):
    """A tensor freed while its own stream has yet to read it: a call on another stream must
    not take its memory."""
    c = SmallCache(ema, [3000], 2, 16, "bf16", seed=47)
    try:
        q = dev16(c.queries(8, 4), "bf16")
        starts, lam = i32([0, 8]), torch.full((2,), 0.5, device="cuda")
        size = ema.paged_prompt_workspace if maps == 1 else ema.paged_diff_prompt_workspace
        n = size(c.h, 8, 1, 4, c.width)
        assert n > 0
        out = torch.empty((8, 4 // maps, 128 * maps), device="cuda")
        side = torch.cuda.Stream()
        kept = torch.empty(n, dtype=torch.uint8, device="cuda")
        x = torch.full((n,), 3, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        kept.copy_(x)
        del x
        if maps == 1:
            ema.paged_prompt_attention(c.h, q, starts, c.table_dev, c.lens_dev, out, stream=side)
        else:
            ema.paged_diff_prompt_attention(c.h, q, starts, c.table_dev, c.lens_dev, lam, out,
                                            stream=side)
        torch.cuda.synchronize()
        assert torch.all(kept == 3)
    finally:
        c.close()


@pytest.mark.parametrize("maps", [1, 2])
@pytest.mark.parametrize("lens,new,H,Hq", [
    ([300, 40], [300, 33], 2, 200),                      # more than 64 tiles of a sequence
    ([70, 9, 200, 33, 1, 90, 0, 150], [70, 3, 150, 33, 1, 0, 0, 66], 2, 8),
    ([70, 9, 200, 33, 1, 90, 0, 150, 81], [70, 3, 150, 33, 1, 0, 0, 66, 80], 2, 8),
])
def test_tiles_of_few_sequences(ema, maps, lens, new, H, Hq):
    c = SmallCache(ema, lens, H, 16, "bf16", seed=48)
    try:
        check_attention(ema, c, new, Hq, "bf16", maps)
        assert ema.slice_device_errors(c.h) == 0
    finally:
        c.close()
