"""Trees of drafted tokens in float64 and plain Python: what the operators of
include/ema_tree.h are checked against.

A request's last n tokens are the nodes of its tree; parents count from its first
row, -1 is a root. A row of tree attention sees every token before the nodes
and those nodes whose bits its mask has.
"""
import numpy as np

from .attention import _gather_sequence
from .layout import to_float64
from .ops import _weights


def tree_tables(parents, starts, seq_lens, words):
    """(mask uint64 [T][words], positions [T], base [B]) for valid input."""
    T = len(parents)
    mask, pos = np.zeros((T, words), np.uint64), np.zeros(T, np.int64)
    base = [int(n) - int(e - s) for n, s, e in zip(seq_lens, starts, starts[1:])]
    for b, (s, e) in enumerate(zip(starts, starts[1:])):
        for row in range(s, e):
            j, depth = row - s, -1
            while j >= 0:
                mask[row, j // 64] |= np.uint64(1) << np.uint64(j % 64)
                j, depth = int(parents[s + j]), depth + 1
            pos[row] = base[b] + depth
    return mask, pos, np.array(base, np.int64)


def tree_accept(parents, starts, drafted, choice, cap, root_choice=None):
    """(path [B][cap], its lengths, the tokens after it)."""
    B = len(starts) - 1
    path, count, after = np.full((B, cap), -1, np.int64), np.zeros(B, np.int64), np.zeros(B, np.int64)
    for b in range(B):
        s, n = int(starts[b]), int(starts[b + 1] - starts[b])
        want, at, k = -1 if root_choice is None else int(root_choice[b]), -1, 0
        while k < cap:
            if root_choice is None and k == 0:
                children = [0] if n else []
            else:
                children = [i for i in range(n) if parents[s + i] == at and drafted[s + i] == want]
            if not children:
                break
            at = path[b, k] = children[0]
            want, k = int(choice[s + at]), k + 1
        count[b], after[b] = k, want
    return path, count, after


def tree_attention(q16, starts, block_table, seq_lens, mask, read_block, kv_heads, head_dim,
                   block_size, dtype, scale=None):
    """q16 uint16 [T][Hq][D], mask uint64 [T][words]. (out, mass) float64 [T][Hq][D]; rows
    outside the starts are NaN."""
    q = to_float64(q16, dtype)
    T, Hq, D = q.shape
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    out, mass = np.full(q.shape, np.nan), np.zeros(q.shape)
    words = mask.shape[1]
    for b, n in enumerate(np.asarray(seq_lens, np.int64)):
        r0, r1 = int(starts[b]), int(starts[b + 1])
        if r1 == r0:
            continue
        out[r0:r1] = 0.0
        if n == 0:
            continue
        base = int(n) - (r1 - r0)
        K16, V16 = _gather_sequence(read_block, block_table[b], int(n), kv_heads, head_dim,
                                    block_size)
        K, V = to_float64(K16, dtype), to_float64(V16, dtype)
        for row in range(r0, r1):
            if base + row - r0 < 0:
                continue
            sees = [t for t in range(int(n)) if t < base or (
                t - base < 64 * words and int(mask[row, (t - base) // 64]) >> ((t - base) % 64) & 1)]
            for h in range(Hq if sees else 0):
                kv = h // (Hq // kv_heads)
                w, v = _weights(q[row, h], K[kv, sees], scale), V[kv, sees]
                out[row, h], mass[row, h] = w @ v, w @ np.abs(v)
    return out, mass


def kv_compact(local, far, far_nhd, tables, base, keep, n_keep, kv_heads, head_dim, block_size):
    """local, far: uint8 [blocks][block_bytes], changed in place; the lengths after it."""
    half = kv_heads * block_size * head_dim
    base, keep = np.asarray(base, np.int64), np.asarray(keep, np.int64)

    def parts(pool, nhd):
        """K and V of a pool's blocks as [block][token][head][channel] views."""
        e = pool.view(np.uint16).reshape(len(pool), 2, half)
        if nhd:
            return [e[:, i].reshape(-1, block_size, kv_heads, head_dim) for i in (0, 1)]
        return [e[:, 0].reshape(-1, kv_heads, block_size, head_dim).transpose(0, 2, 1, 3),
                e[:, 1].reshape(-1, kv_heads, head_dim, block_size).transpose(0, 3, 1, 2)]

    pools = [parts(local, False), parts(far, far_nhd)]

    def at(l, b, t):
        u = int(tables[l, b, t // block_size])
        return (0, u, t % block_size) if u < len(local) else (1, u - len(local), t % block_size)

    for l in range(len(tables)):
        for b in range(len(base)):
            for k in range(int(n_keep[b])):
                src, dst = at(l, b, int(base[b] + keep[b, k])), at(l, b, int(base[b] + k))
                for i in (0, 1):
                    pools[dst[0]][i][dst[1], dst[2]] = pools[src[0]][i][src[1], src[2]]
    return base + np.asarray(n_keep, np.int64)
