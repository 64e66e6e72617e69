"""Every form of tree attention against 64 bits: rows of an item (64, 128, 256, several items),
block sizes, types, weights in one and in several parts, items that stay whole and items
that are shared, join records kept by item and by workgroup; values and keys that are not
finite in each; bad starts that ask for more work than the sizes allow for."""
import numpy as np
import pytest
import torch

from harness import TORCH_DT
from ops_harness import D, assert_close, dev16, i32, scores_bounded
from oracle import attention as oattn
from oracle import to_float64
from test_gpu_tree import Case, full

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


def attends(k, b):
    """[node][token] of request b: which tokens a node attends."""
    s, e = int(k.starts[b]), int(k.starts[b + 1])
    n = int(k.c.lens[b])
    t = np.arange(n) - (n - (e - s))
    bits = k.mask[s:e][:, np.clip(t, 0, None) // 64] >> (np.clip(t, 0, None) % 64).astype(np.uint64)
    return (t < 0) | (bits & np.uint64(1)).astype(bool)


def keys_and_values(k, b):
    c = k.c
    K, V = oattn._gather_sequence(c.read_block, c.table[b], int(c.lens[b]), k.heads[1], D, c.bs)
    return to_float64(K, k.dtype), to_float64(V, k.dtype)


def dense(k):
    """(out, mass) in float64, a request and KV head at a time."""
    Hq, H = k.heads
    q = to_float64(k.q16, k.dtype)
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(len(k.c.lens)):
        s, e = int(k.starts[b]), int(k.starts[b + 1])
        if e == s:
            continue
        sees, (K, V) = attends(k, b), keys_and_values(k, b)
        for h in range(Hq):
            kv = h // (Hq // H)
            x = np.where(sees, q[s:e, h] @ K[kv].T / np.sqrt(D), -np.inf)
            top = x.max(1, keepdims=True)
            w = np.exp(x - np.where(np.isfinite(top), top, 0.0))
            w /= np.maximum(w.sum(1, keepdims=True), 1e-300)
            out[s:e, h], mass[s:e, h] = w @ V[kv], w @ np.abs(V[kv])
    return out, mass


def check(k, got):
    want, mass = dense(k)
    assert_close(got, want, mass, got.dtype, k.dtype, int(k.c.lens.max()))


def test_the_dense_form_is_the_oracle_s(ema):
    k = Case(ema, [90, 7, 200], [20, 7, 70], (4, 2), 16, "bf16", seed=1)
    try:
        for a, b in zip(dense(k), k.ref()):
            assert np.allclose(a, b, rtol=1e-9, atol=1e-12)
    finally:
        k.close()


# mean nodes times 4 heads: 64, 128, 256 rows, several items of 256
NODES = [5, 20, 45, 150]


def sizes(n, whole):
    """Tables of up to 512 tokens are not shared; of the others an item's 24 tiles are."""
    return ([460, n + 1, 130 + n, 500] if whole else [700, n + 3, 1500, 333]), [n, n - 2, n + 3, n]


@pytest.mark.parametrize("parts", ["one", "several"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bs", [16, 32, 64, 128])
@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("n", NODES)
def test_every_form(ema, n, whole, bs, dtype, parts):
    lens, new = sizes(n, whole)
    k = Case(ema, lens, new, (8, 2), bs, dtype, seed=n + bs, extra_width=0 if whole else 1)
    try:
        scores_bounded(k.c, k.q16)
        assert (k.c.width * bs <= 512) == whole
        if parts == "one":
            check(k, k.call(k.out(TORCH_DT[dtype])))
        else:
            got = k.call(k.out(torch.float32))
            check(k, got)
            # rounded once from the same 32 bits
            same = k.call(k.out(TORCH_DT[dtype]), full_weights=True)
            assert torch.equal(same, got.to(TORCH_DT[dtype]))
        assert ema.slice_device_errors(k.c.h) == 0
    finally:
        k.close()


@pytest.mark.parametrize("B,heads,n", [
    (128, (16, 8), 1),        # 1024 items at most, twice the workgroups: records by item
    (129, (16, 8), 1),        # 1032: by workgroup
    (130, (64, 8), 9),        # 128 rows: 1624, by workgroup
    (140, (64, 4), 9),        # 256 rows: 872 of 256 workgroups
])
def test_many_uneven_requests_share_their_items(ema, B, heads, n):
    """A few long requests among short ones: shares of all tiles, several items to each."""
    lens = [1500 if b % 14 == 0 else 20 for b in range(B)]
    k = Case(ema, lens, [n] * B, heads, 16, "bf16", seed=B)
    try:
        check(k, k.call(k.out(torch.float32)))
        check(k, k.call(k.out(torch.bfloat16)))
        assert ema.slice_device_errors(k.c.h) == 0
    finally:
        k.close()


@pytest.mark.parametrize("out", ["f32", "same"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("n", NODES)
def test_values_that_are_not_finite(ema, n, whole, dtype, out):
    inf, nan = {"bf16": (0x7F80, 0x7FC0), "f16": (0x7C00, 0x7E00)}[dtype]
    lens, new = sizes(n, whole)
    k = Case(ema, lens, new, (8, 2), 16, dtype, seed=n, kind="random", extra_width=0 if whole else 1)
    try:
        c, rng = k.c, k.c.rng
        want = np.ones((k.T, 8, D), bool)
        for b in range(4):
            s, base, sees = int(k.starts[b]), lens[b] - new[b], attends(k, b)
            for x in range(6):
                # of nodes, the last older tokens and far ones; heads and channels in turn
                t = base + int(rng.integers(0, new[b])) if x < 4 else int(rng.integers(0, base))
                half, head, ch = int(x == 3), x % 2, int(rng.integers(0, D))
                c.poke(half ^ 1, b, t, head, ch, inf if x % 3 == 0 and not half else nan)
                who = np.flatnonzero(sees[:, t])
                for r in who:
                    if half:                             # NaN in K: the row
                        want[s + r, 4 * head:4 * head + 4] = False
                    else:
                        want[s + r, 4 * head:4 * head + 4, ch] = False
        c.upload()
        got = k.call(k.out(torch.float32 if out == "f32" else TORCH_DT[dtype]))
        assert np.array_equal(torch.isfinite(got).cpu().numpy(), want)
        # the others are as if those were 0: nobody that is left attends them
        e, exponent = c.local.view(np.uint16), 0x7F80 if dtype == "bf16" else 0x7C00
        e[(e & exponent) == exponent] = 0
        ref, mass = dense(k)
        live = torch.from_numpy(want).cuda()
        assert_close(torch.where(live, got, 0), np.where(want, ref, 0), np.where(want, mass, 0),
                     got.dtype, dtype, max(lens))
    finally:
        k.close()


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("n", NODES)
def test_keys_that_are_infinite(ema, n, whole):
    """A score of -inf is no weight, one of +inf makes the row NaN."""
    lens, new = sizes(n, whole)
    k = Case(ema, lens, new, (8, 2), 16, "bf16", seed=n + 1, kind="random", extra_width=0 if whole else 1)
    try:
        c = k.c
        k.q16[:, :, 7] = 0x3F80                          # 1.0
        gone = np.zeros((k.T, 8), bool)
        for b in range(4):
            base, s = lens[b] - new[b], int(k.starts[b])
            c.poke(0, b, base, 0, 7, 0xFF80)             # its first node, of one KV head
            c.poke(0, b, base // 2, 1, 7, 0xFF80)        # an older token, of the other
            c.poke(0, b, base + new[b] - 1, 1, 7, 0x7F80)     # its last node: +inf
            gone[s:s + new[b], 4:] = attends(k, b)[:, lens[b] - 1, None]
        c.upload()
        got = k.call(k.out(torch.float32))
        with np.errstate(all="ignore"):
            want, mass = dense(k)
        assert torch.isnan(got[torch.from_numpy(gone).cuda()]).all()
        live = np.broadcast_to(~gone[:, :, None], want.shape)
        assert np.isfinite(want[live]).all()
        assert_close(torch.where(torch.from_numpy(live.copy()).cuda(), got, 0), np.where(live, want, 0),
                     np.where(live, mass, 0), torch.float32, "bf16", max(lens))
    finally:
        k.close()


def test_more_units_than_32_bits_hold(ema):
    """Starts that give every second of 40000 requests all rows: 20000 * 1024 items of 160 units
    each, 3.3e9. The call ends without them; the requests are counted."""
    B, T, G, bs = 40000, 1024, 64, 256
    h = ema.slice_create(1, D, bs, "bf16", 0, 4 * 2 * bs * D * 2, 0)
    try:
        starts = np.zeros(B + 1, np.int64)
        starts[1::2] = T
        q = torch.zeros((T, G, D), dtype=torch.bfloat16, device="cuda")
        out = torch.full((T, G, D), 7.0, dtype=torch.bfloat16, device="cuda")
        ema.paged_tree_attention(h, q, i32(starts), torch.zeros((B, 39), dtype=torch.int32, device="cuda"),
                                 full((B,), 39 * bs), full((T, 16), -1, torch.int64), out)
        assert ema.slice_device_errors(h) == B // 2
        assert (out == 7).all()
    finally:
        torch.cuda.synchronize()
        ema.slice_destroy(h)
