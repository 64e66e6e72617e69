"""Small paged caches with scattered blocks for the operator tests: every row
that no request owns holds NaN, so that a read past a length shows.

Tolerances. A 16-bit output is off by at most half a step of its value, and
its softmax weights, rounded once to 16 bits, by half a step of each, which
moves the output by at most that times the row's mass (sum of |weight| |value|).
float16 weights below 2^-14 are off by up to 2^-25 of the largest weight (at most
the sum of weights) each. Scores: 128 products of exact 16-bit values summed in 32
bits, each partial sum off by at most 2^-24 of its size, which stays below 32 after
scaling here (checked), so a score is off by at most 128 * 2^-24 * 32 = 2.5e-4 and
a weight by e^(2 * 2.5e-4) - 1; rounding errors that all point one way do not
occur, and a tenth of it is allowed: 5e-5. A norm doubles what a weight's error
does (the row and its mean square)."""
import numpy as np
import torch

import synth
from harness import TORCH_DT
from oracle.layout import to_float64

D = 128
WEIGHT_ERR = 5e-5
NAN16 = synth.NAN16


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device="cuda")


def dev16(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(TORCH_DT[dtype])


class SmallCache:
    """A local pool with the requests' tokens in scattered blocks."""

    def __init__(self, ema, lens, kv_heads, block_size, dtype, seed=0, spare=3, extra_width=1,
                 checked=False, n_slice=0):
        self.ema, self.dtype, self.H, self.bs = ema, dtype, kv_heads, block_size
        self.rng = rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens, np.int64)
        nblk = -(-self.lens // block_size)
        self.n_local = int(nblk.sum()) + spare
        self.width = int(nblk.max(initial=0)) + extra_width
        bb = 2 * block_size * kv_heads * D * 2
        self.h = ema.slice_create(kv_heads, D, block_size, dtype, 0, self.n_local * bb,
                                  n_slice * bb, checked=checked)
        ids = rng.permutation(self.n_local)
        self.table = np.full((len(self.lens), self.width), -1, np.int64)
        e = np.full((self.n_local, bb // 2), NAN16[dtype], np.uint16)
        at = 0
        for b, n in enumerate(self.lens):
            mine = ids[at:at + nblk[b]]
            at += nblk[b]
            self.table[b, :nblk[b]] = mine
            for j, u in enumerate(mine):
                t = min(block_size, int(n) - j * block_size)
                for half in (0, 1):
                    h, tt, d = np.meshgrid(np.arange(kv_heads), np.arange(t), np.arange(D),
                                           indexing="ij")
                    e[u, synth.element_index(0, half, h, tt, d, kv_heads, block_size, D)] = \
                        synth.random_16bit(rng, h.shape, dtype)
        self.local = e.view(np.uint8).reshape(self.n_local, bb)
        self.view = ema.pool_view(self.h, ema.POOL_LOCAL)
        self.upload()
        self.table_dev, self.lens_dev = i32(self.table), i32(self.lens)

    def upload(self):
        self.view.copy_(torch.from_numpy(self.local))
        torch.cuda.synchronize()

    def read_block(self, u):
        return self.local[u]

    def element(self, half, b, t, h):
        """Element indices (block, elements) of token t of request b, head h."""
        u = self.table[b, t // self.bs]
        d = np.arange(D)
        return u, synth.element_index(0, half, h, t % self.bs, d, self.H, self.bs, D)

    def poke(self, half, b, t, h, channel, pattern):
        """One element of K or V set to a 16-bit pattern (not uploaded)."""
        u, e = self.element(half, b, t, h)
        self.local.view(np.uint16).reshape(self.n_local, -1)[u, e[channel]] = pattern

    def queries(self, n, q_heads):
        return synth.random_16bit(self.rng, (n, q_heads, D), self.dtype)

    def close(self):
        self.view = None
        torch.cuda.synchronize()
        self.ema.slice_destroy(self.h)


def scores_bounded(cache, q16):
    """The inputs stay within what the tolerance of the scores assumes."""
    q = to_float64(q16, cache.dtype)
    e = to_float64(cache.local.view(np.uint16), cache.dtype)
    kmax = np.nanmax(np.abs(e[np.isfinite(e)]), initial=0.0)
    rms = np.sqrt(np.mean(e[np.isfinite(e)] ** 2)) if np.isfinite(e).any() else 0.0
    worst = np.linalg.norm(q, axis=-1).max(initial=0.0) * rms * 6 / np.sqrt(D)
    assert worst <= 32 and kmax <= 16


def assert_close(got, ref, mass, out_dtype, cache_dtype, n, norm=False):
    """got: torch tensor; ref, mass from the oracle; n: the longest request."""
    x = got.double().cpu().numpy()
    half = 0.0 if out_dtype == torch.float32 else torch.finfo(out_dtype).eps / 2
    w = WEIGHT_ERR
    if out_dtype != torch.float32:
        w += torch.finfo(TORCH_DT[cache_dtype]).eps / 2
    tiny = n * 2.0 ** -25 * 6 if cache_dtype == "f16" and out_dtype != torch.float32 else 0.0
    scale = mass.max(axis=-1, keepdims=True) if norm else mass
    tol = half * np.abs(ref) + (2 if norm else 1) * (w * scale + tiny * (scale > 0)) + 1e-30
    live = ~np.isnan(ref)
    assert np.isfinite(x[live]).all()
    bad = np.abs(x - ref) > tol * (1 + half)
    bad &= live
    assert not bad.any(), (int(bad.sum()), float((np.abs(x - ref) / tol)[live].max()))
