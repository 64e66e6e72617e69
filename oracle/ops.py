"""Tables of a step, the store of a chunk's tokens, and attention of prompt
chunks (plain and differential) in float64: what the operators of
include/ema_ops.h are checked against.

Positions: request b has len_b tokens, the last new_b of them new; the i-th new
one sits at len_b - new_b + i and attends to every token up to itself.

    plain          o = sum_t w_t v_t, w = softmax(scale q . k_t)
    differential   o = sum_t (w1_t - lambda w2_t) v_t, the maps' queries and keys
                   in heads 2i, 2i + 1, v the two KV heads side by side;
                   optionally o / sqrt(mean(o^2) + eps) * weight

Beside each output row comes its mass, sum_t |weights|_t |v_t| per channel: a
relative error e of the weights moves the output by at most e * mass.
"""
import numpy as np

from .layout import to_float64
from .attention import _gather_sequence


def kv_tables(block_ids, seq_lens, new_lens, max_blocks, block_size, n_local, n_slots,
              staging=None, writeback_cap=0):
    """Everything ema_kv_tables writes, as a dict of int arrays, for valid input."""
    ids = np.asarray(block_ids, np.int64)
    L, B = ids.shape[0], len(seq_lens)
    canon = np.full((L, B, max_blocks), -1, np.int64)
    table = canon.copy()
    starts = np.concatenate([[0], np.cumsum(new_lens)]).astype(np.int64)
    slots = np.full((L, n_slots), -1, np.int64)
    stage_n = 0 if staging is None else staging.shape[1]
    pf = [np.full((L, stage_n), -1, np.int64) for _ in range(2)] + [np.zeros(L, np.int64)]
    wb = [np.full((L, writeback_cap), -1, np.int64) for _ in range(2)] + [np.zeros(L, np.int64)]
    for l in range(L):
        f = r = 0
        for b in range(B):
            n, old = int(seq_lens[b]), int(seq_lens[b]) - int(new_lens[b])
            for j in range(-(-n // block_size)):
                u = int(ids[l, f])
                f += 1
                canon[l, b, j] = table[l, b, j] = u
                if u >= n_local and staging is not None:
                    s = table[l, b, j] = int(staging[l % staging.shape[0], r])
                    r += 1
                    first, end = j * block_size, (j + 1) * block_size
                    for lists, yes, src, dst in ((pf, first < old, u, s),
                                                 (wb, end > old and n > old, s, u)):
                        if yes:
                            k = lists[2][l]
                            lists[0][l, k], lists[1][l, k] = src, dst
                            lists[2][l] += 1
            for i in range(n - old):
                u = table[l, b, (old + i) // block_size]
                if 0 <= u < n_local:
                    slots[l, starts[b] + i] = u * block_size + (old + i) % block_size
    return {"canon": canon, "table": table, "starts": starts, "slots": slots,
            "prefetch": pf, "writeback": wb}


def kv_store(local, k16, v16, slots, kv_heads, head_dim, block_size):
    """local: uint8 [n_local][block_bytes], changed in place; k16, v16 uint16
    [T][Hkv][D]; slots int [T], -1: not stored."""
    half = kv_heads * block_size * head_dim
    e = local.view(np.uint16).reshape(len(local), 2, half)
    K = e[:, 0].reshape(-1, kv_heads, block_size, head_dim)
    V = e[:, 1].reshape(-1, kv_heads, head_dim, block_size)
    for t, s in enumerate(np.asarray(slots, np.int64)):
        if s >= 0:
            K[s // block_size, :, s % block_size] = k16[t]
            V[s // block_size, :, :, s % block_size] = v16[t]


def _weights(q, K, scale):
    s = (K @ q) * scale
    w = np.exp(s - s.max())
    return w / w.sum()


def prompt_attention(q16, starts, block_table, seq_lens, read_block, kv_heads, head_dim,
                     block_size, dtype, scale=None, lam=None, norm_weight=None, norm_eps=0.0):
    """q16 uint16 [T][Hq][D]; lam given: differential. Returns (out, mass), float64
    [T][heads][channels]; rows outside [starts[0], starts[-1]) are NaN."""
    q = to_float64(q16, dtype)
    T, Hq, D = q.shape
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    maps = 1 if lam is None else 2
    out = np.full((T, Hq // maps, maps * D), np.nan)
    mass = np.zeros_like(out)
    G = Hq // kv_heads
    for b, n in enumerate(np.asarray(seq_lens, np.int64)):
        r0, r1 = int(starts[b]), int(starts[b + 1])
        if r1 == r0:
            continue
        out[r0:r1] = 0.0
        if n == 0:
            continue
        K16, V16 = _gather_sequence(read_block, block_table[b], int(n), kv_heads, head_dim,
                                    block_size)
        K, V = to_float64(K16, dtype), to_float64(V16, dtype)
        for row in range(r0, r1):
            seen = int(n) - (r1 - row) + 1
            if seen <= 0:
                continue
            for h in range(Hq // maps):
                kv = maps * (h // G)
                w = _weights(q[row, maps * h], K[kv, :seen], scale)
                v = V[kv, :seen]
                a = w
                if maps == 2:
                    w2 = lam[h] * _weights(q[row, 2 * h + 1], K[kv + 1, :seen], scale)
                    v = np.concatenate([v, V[kv + 1, :seen]], axis=1)
                    w, a = w - w2, w + np.abs(w2)
                o, m = w @ v, a @ np.abs(v)
                if norm_weight is not None:
                    rms = np.sqrt((o ** 2).mean() + norm_eps)
                    o, m = o / rms * norm_weight, m / rms * np.abs(norm_weight)
                out[row, h], mass[row, h] = o, m
    return out, mass
