"""The operators of decoding with drafted trees over a paged cache, as cases to
measure, with their plain forms.

  tables   ancestor masks, positions and first places of drafted trees
  tree     attention of the trees' nodes over the paged cache
  accept   the path of a tree that the model's choices confirm
  compact  kept tokens moved together in the cache, all layers

A request's drafted tokens are its last ones. The shapes are those of
``synth/configs.py`` (a tiny MHA cache, an 8B-shaped GQA cache, one GPU's share of
a 70B-shaped cache) and generic ones around them. Lengths are evenly spaced
quantiles of the case's ranges in a seeded order, so the work of a case does not
depend on the seed; trees, placements and values do.
"""
import math

import numpy as np
import torch

own = False

D = 128
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
VOCAB = 32000


def listed():
    return [
        # one request with a small tree: all latency
        {"name": "tables-one", "op": "tables", "block": 16, "batch": 1, "ctx_lo": 999,
         "ctx_hi": 999, "new_lo": 15, "new_hi": 15, "forest": 0},
        # a step of many requests with trees of several mask words
        {"name": "tables-wide", "op": "tables", "block": 16, "batch": 200, "ctx_lo": 0,
         "ctx_hi": 4000, "new_lo": 65, "new_hi": 250, "forest": 1},
        # three short requests of an MHA cache, the result kept in 32 bits
        {"name": "tree-tiny", "op": "tree", "q_heads": 8, "kv_heads": 8, "block": 16,
         "dtype": "f16", "out": "f32", "batch": 3, "ctx_lo": 0, "ctx_hi": 101, "new_lo": 1,
         "new_hi": 13, "forest": 1},
        # a verification step of the 8B-shaped cache: the decode batch, small trees
        {"name": "tree-8b", "op": "tree", "q_heads": 32, "kv_heads": 8, "block": 16,
         "dtype": "bf16", "out": "bf16", "batch": 64, "ctx_lo": 1024, "ctx_hi": 4080,
         "new_lo": 16, "new_hi": 16, "forest": 0},
        # fewer requests of that layer, wide ragged trees
        {"name": "tree-8b-wide", "op": "tree", "q_heads": 32, "kv_heads": 8, "block": 16,
         "dtype": "bf16", "out": "bf16", "batch": 16, "ctx_lo": 500, "ctx_hi": 8001,
         "new_lo": 48, "new_hi": 64, "forest": 0},
        # one long document on one GPU's share of a 70B-shaped layer
        {"name": "tree-70b-long", "op": "tree", "q_heads": 8, "kv_heads": 1, "block": 32,
         "dtype": "bf16", "out": "bf16", "batch": 1, "ctx_lo": 32001, "ctx_hi": 32001,
         "new_lo": 31, "new_hi": 31, "forest": 0},
        # drafts of more nodes than a mask word, large blocks
        {"name": "tree-large", "op": "tree", "q_heads": 16, "kv_heads": 4, "block": 64,
         "dtype": "f16", "out": "f16", "batch": 5, "ctx_lo": 2001, "ctx_hi": 9001,
         "new_lo": 33, "new_hi": 131, "forest": 1},
        # the choices of one request against its tree
        {"name": "accept-one", "op": "accept", "block": 16, "batch": 1, "ctx_lo": 99,
         "ctx_hi": 99, "new_lo": 7, "new_hi": 7, "forest": 0, "cap": 4},
        # a large decode batch
        {"name": "accept-batch", "op": "accept", "block": 16, "batch": 256, "ctx_lo": 99,
         "ctx_hi": 99, "new_lo": 31, "new_hi": 64, "forest": 1, "cap": 10},
        # one request, one layer, two accepted tokens
        {"name": "compact-one", "op": "compact", "layers": 1, "kv_heads": 8, "block": 16,
         "dtype": "f16", "layout": "attn", "slice": 0.0, "batch": 1, "ctx_lo": 50, "ctx_hi": 50,
         "new_lo": 7, "new_hi": 7, "keep_pct": 30, "head": 1},
        # accepted paths of the decode batch in all layers of the 8B-shaped cache, 30 % of it in
        # the slice
        {"name": "compact-8b", "op": "compact", "layers": 32, "kv_heads": 8, "block": 16,
         "dtype": "bf16", "layout": "attn", "slice": 0.3, "batch": 64, "ctx_lo": 0, "ctx_hi": 200,
         "new_lo": 16, "new_hi": 16, "keep_pct": 25, "head": 1},
        # long contexts thinned to half of their tokens, a 70B share with a token-major slice
        {"name": "compact-thin", "op": "compact", "layers": 80, "kv_heads": 1, "block": 32,
         "dtype": "bf16", "layout": "nhd", "slice": 0.5, "batch": 8, "ctx_lo": 0, "ctx_hi": 0,
         "new_lo": 901, "new_hi": 3501, "keep_pct": 50, "head": 4},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_FLOPS, MOST_BYTES, MOST_SCORES, MOST_POOL, MOST_ABOVE = 6e10, 6.8e8, 1.1e9, 1.4e9, 4e7


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        if w["flops"] > MOST_FLOPS or w["bytes"] > MOST_BYTES:
            continue
        pairs = _pairs(c)
        if c["op"] in ("tables", "accept") and len(pairs) * max(n for _, n in pairs) ** 2 > MOST_ABOVE:
            continue
        if c["op"] == "tree" and len(pairs) * c["q_heads"] * max(n for _, n in pairs) * max(
                x + n for x, n in pairs) > MOST_SCORES:       # the plain form's padded scores
            continue
        if c["op"] == "compact" and c["layers"] * sum(_blocks(c, pairs)) * _block_bytes(c) > MOST_POOL:
            continue
        return c


def _draw(rng):
    op = rng.choice(["tables", "tree", "tree", "tree", "tree", "accept", "compact", "compact"])
    c = {"op": op, "block": rng.choice([16, 16, 32, 64, 128, 256]), "forest": rng.choice([0, 1])}
    if op in ("tree", "compact"):
        c["dtype"] = rng.choice(["bf16", "f16"])
        c["kv_heads"] = rng.choice([1, 2, 4, 8, 8])
    if op == "tree":
        c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 3, 4, 4, 7, 8])
        c["out"] = rng.choice([c["dtype"], c["dtype"], c["dtype"], "f32"])
    if op == "compact":
        del c["forest"]
        c["layers"] = _log(rng, 1, 80)
        c["layout"] = rng.choice(["attn", "nhd"])
        c["slice"] = rng.choice([0.0, 0.3, 0.5, 0.9])
        c["batch"] = _log(rng, 1, 64)
        c["keep_pct"] = rng.choice([10, 25, 50, 90])
        c["head"] = rng.choice([0, 1, 4])
        long = rng.random() < 0.35           # a context thinned out, else a draft's path
        c["new_hi"] = _log(rng, 64, 4000) if long else _log(rng, 8, 128)
        c["new_lo"] = max(8, int(c["new_hi"] * rng.choice([0.3, 1.0])))
    elif op == "tree":
        c["batch"] = _log(rng, 1, 96)
        c["new_hi"] = _log(rng, 1, 256)
        c["new_lo"] = 1 + int((c["new_hi"] - 1) * rng.choice([0.0, 0.5, 1.0, 1.0]))
    else:
        c["batch"] = _log(rng, 1, 600)
        c["new_hi"] = _log(rng, 8 if op == "tables" else 1, 1000)
        c["new_lo"] = 1 + int((c["new_hi"] - 1) * rng.choice([0.0, 0.5, 1.0]))
        if op == "accept":
            c["cap"] = min(c["new_hi"], _log(rng, 1, 24))
    most = {"tree": 30000, "compact": 300}.get(op, 3000)
    c["ctx_hi"] = rng.choice([0, _log(rng, 1, most), _log(rng, 1, most)])
    c["ctx_lo"] = int(c["ctx_hi"] * rng.choice([0.0, 0.5, 1.0]))
    return c


# ---- lengths and work ------------------------------------------------------------

def _spread(lo, hi, n):
    return [lo if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _pairs(c):
    """(tokens before the tree, its nodes) of every sequence, independent of the seed."""
    B = c["batch"]
    ctx, new = _spread(c["ctx_lo"], c["ctx_hi"], B), _spread(c["new_lo"], c["new_hi"], B)
    return [(ctx[i * 7 % B] if B % 7 else ctx[i], new[i]) for i in range(B)]


def _blocks(c, pairs):
    return [-(-(x + n) // c["block"]) for x, n in pairs]


def _block_bytes(c):
    return 2 * c["block"] * c["kv_heads"] * D * 2


def _itemsize(t):
    return 4 if t == "f32" else 2


def _words(pairs):
    return -(-max(n for _, n in pairs) // 64)


def _kept(c, n):
    """Tokens that a request of n keeps; its first c["head"] stay in place, all others move."""
    return max(c["head"], min(n - 1, max(1, n * c["keep_pct"] // 100)))


def work(c):
    pairs = _pairs(c)
    B, T = len(pairs), sum(n for _, n in pairs)
    if c["op"] == "tables":
        # parents, starts and lengths in; masks, positions and first places out
        return {"bytes": 4 * (T + B + 1 + B) + 8 * T * _words(pairs) + 4 * (T + B), "flops": 0}
    if c["op"] == "accept":
        # parents, drafted tokens, choices, starts in; paths, their lengths, next tokens out
        return {"bytes": 4 * (3 * T + B + 1 + (B if c["forest"] else 0) + B * c["cap"] + 2 * B),
                "flops": 0}
    if c["op"] == "compact":
        kept = [_kept(c, n) for _, n in pairs]
        moved = sum(k - c["head"] for k in kept)
        b = 2 * moved * c["layers"] * c["kv_heads"] * 2 * D * 2
        return {"bytes": b + 4 * (sum(kept) + 3 * B), "flops": 0}
    Hq = c["q_heads"]
    b = 4 * (B + 1 + B + sum(_blocks(c, pairs))) + T * Hq * D * (2 + _itemsize(c["out"]))
    b += 8 * T * _words(pairs) + sum(x + n for x, n in pairs) * 2 * c["kv_heads"] * D * 2
    # per node, head and token: q.k and the weighted V; of its tree a node attends itself at least
    return {"bytes": b, "flops": 4 * D * Hq * sum(n * (x + 1) for x, n in pairs)}


# ---- inputs ----------------------------------------------------------------------

class _State:
    """What a program keeps between calls; with the framework, also the slice
    handle that owns the pools."""
    h = None

    def close(self):
        if self.h is not None:
            from paper_2609_27040_amd import ema
            self.pool = self.far = None
            ema.slice_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def _normal(g, shape, dt, factor=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * factor).to(dt)


def _tree(rng, n, forest):
    """Parents of n nodes, in the order of a draft: chains with branches; one root, or several."""
    i = np.arange(n)
    back = 1 + rng.geometric(0.3, n)
    p = np.where(rng.random(n) < 0.4, i - 1, i - back)
    p = np.maximum(p, -1 if forest else 0)
    p[0] = -1
    return p


def _inputs(c, seed, S):
    """Everything of a case but the pools' place, from the seed alone."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    pairs = _pairs(c)
    pairs = [pairs[i] for i in rng.permutation(len(pairs))]
    S.case, S.pairs, S.bs = c, pairs, c["block"]
    S.B, S.T, S.most = len(pairs), sum(n for _, n in pairs), max(n for _, n in pairs)
    lens = np.array([x + n for x, n in pairs], dtype=np.int32)
    new = np.array([n for _, n in pairs], dtype=np.int32)
    S.new = new
    i32 = dict(dtype=torch.int32, device="cuda")
    if c["op"] == "compact":
        _compact_inputs(c, rng, S, lens, new)
        return g
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    S.seq_lens, S.query_start = _gpu(lens), _gpu(starts)
    trees = [_tree(rng, n, c["forest"]) for n in new]
    parents = np.concatenate(trees).astype(np.int32)
    S.parents, S.words = _gpu(parents), _words(pairs)
    if c["op"] == "tables":
        S.mask = torch.empty((S.T, S.words), dtype=torch.int64, device="cuda")
        S.positions, S.base = torch.empty(S.T, **i32), torch.empty(S.B, **i32)
        return g
    if c["op"] == "accept":
        drafted = rng.integers(0, VOCAB, S.T).astype(np.int32)
        choice = rng.integers(0, VOCAB, S.T).astype(np.int32)
        root = rng.integers(0, VOCAB, S.B).astype(np.int32)
        # seven times of ten the model's choice is one of the drafted children
        child = np.flatnonzero(rng.random(S.T) < 0.7)
        b = np.repeat(np.arange(S.B), new)[child]
        up = parents[child]
        inner = up >= 0
        choice[starts[b[inner]] + up[inner]] = drafted[child[inner]]
        root[b[~inner]] = drafted[child[~inner]]
        S.drafted, S.choice = _gpu(drafted), _gpu(choice)
        S.root_choice = _gpu(root) if c["forest"] else None
        S.path = torch.empty((S.B, c["cap"]), **i32)
        S.n_path, S.next = torch.empty(S.B, **i32), torch.empty(S.B, **i32)
        return g
    S.H, S.Hq, S.dt = c["kv_heads"], c["q_heads"], DT[c["dtype"]]
    nblk = np.array(_blocks(c, pairs))
    S.nb, S.width = int(nblk.sum()) + 3, int(nblk.max())
    first = np.concatenate([[0], np.cumsum(nblk)])
    ids = rng.permutation(S.nb)[:first[-1]]
    S.mask = _gpu(np.concatenate([_bits(t, S.words) for t in trees]).view(np.int64))
    table = np.full((S.B, S.width), -1, dtype=np.int32)
    for b in range(S.B):
        table[b, :nblk[b]] = ids[first[b]:first[b + 1]]
    S.block_table = _gpu(table)
    S.q = _normal(g, (S.T, S.Hq, D), S.dt, 1.5)
    S.out = torch.empty((S.T, S.Hq, D), dtype=DT[c["out"]], device="cuda")
    return g


def _bits(parents, words):
    """Ancestor masks of one tree, uint64 [n][words]."""
    m = np.zeros((len(parents), words), dtype=np.uint64)
    for i, p in enumerate(parents):
        if p >= 0:
            m[i] = m[p]
        m[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return m


def _compact_inputs(c, rng, S, lens, new):
    L, S.H, S.dt = c["layers"], c["kv_heads"], DT[c["dtype"]]
    nblk = np.array(_blocks(c, S.pairs))
    N, S.width = int(nblk.sum()), int(nblk.max())
    far = int(math.floor(c["slice"] * N + 0.5))
    S.n_local, S.n_far = L * (N - far) + 1, L * far
    local, away = rng.permutation(S.n_local)[:L * (N - far)], rng.permutation(S.n_far) + S.n_local
    first = np.concatenate([[0], np.cumsum(nblk)])
    table = np.full((L, S.B, S.width), -1, dtype=np.int32)
    for l in range(L):
        ids = np.concatenate([local[l * (N - far):(l + 1) * (N - far)], away[l * far:(l + 1) * far]])
        ids = rng.permutation(ids)
        for b in range(S.B):
            table[l, b, :nblk[b]] = ids[first[b]:first[b + 1]]
    kept = np.array([_kept(c, n) for n in new])
    keep = np.full((S.B, kept.max()), -1, dtype=np.int32)
    head = c["head"]
    for b, n in enumerate(new):
        keep[b, :head] = np.arange(head)
        rest = head + 1 + rng.permutation(n - head - 1)[:kept[b] - head]
        keep[b, head:kept[b]] = np.sort(rest)
    S.table, S.keep, S.n_keep = _gpu(table), _gpu(keep), _gpu(kept.astype(np.int32))
    S.base = _gpu(lens - new)
    S.new_lens = torch.empty(S.B, dtype=torch.int32, device="cuda")


def _fill(g, pool, blocks, dt):
    """Values of a pool's first blocks, the same whoever owns it."""
    flat = pool[:blocks].view(-1).view(dt)
    for s in range(0, flat.numel(), 1 << 27):
        e = min(flat.numel(), s + (1 << 27))
        flat[s:e].copy_(torch.randn(e - s, generator=g, device="cuda"))


def prepare(case, seed):
    S = _State()
    g = _inputs(case, seed, S)
    S.far = None
    if case["op"] in ("tables", "accept"):
        if own:
            from paper_2609_27040_amd import ema
            bb = 2 * S.bs * D * 2                # one KV head: the trees do not depend on it
            S.h = ema.slice_create(1, D, S.bs, "bf16", ema.LAYOUT_ATTN, 4 * bb, 0)
        return S
    bb = _block_bytes(case)
    local, far = (S.n_local, S.n_far) if case["op"] == "compact" else (S.nb, 0)
    if own:
        from paper_2609_27040_amd import ema
        layout = ema.LAYOUT_NHD if case.get("layout") == "nhd" else ema.LAYOUT_ATTN
        S.h = ema.slice_create(S.H, D, S.bs, case["dtype"], layout, local * bb, far * bb)
        S.pool = ema.pool_view(S.h, ema.POOL_LOCAL)
        S.far = ema.pool_view(S.h, ema.POOL_SLICE) if far else None
    else:
        # one block more, where a plain scatter puts what goes to the other pool
        S.pool = torch.empty((local + 1, bb), dtype=torch.uint8, device="cuda")
        S.far = torch.empty((far + 1, bb), dtype=torch.uint8, device="cuda") if far else None
    _fill(g, S.pool, local, S.dt)
    if far:
        _fill(g, S.far, far, S.dt)
    return S


# ---- one pass ----------------------------------------------------------------------

def run(S):
    op = S.case["op"]
    if own:
        from paper_2609_27040_amd import ema
        if op == "tables":
            ema.tree_tables(S.h, S.parents, S.query_start, S.seq_lens, S.mask, S.positions, S.base)
            return [S.mask, S.positions, S.base]
        if op == "accept":
            ema.tree_accept(S.h, S.parents, S.query_start, S.drafted, S.choice, S.path, S.n_path,
                            S.next, root_choice=S.root_choice)
            return [S.path, S.n_path, S.next]
        if op == "compact":
            ema.kv_compact(S.h, S.table, S.base, S.keep, S.n_keep, new_lens=S.new_lens)
            return _pools(S, S.new_lens)
        ema.paged_tree_attention(S.h, S.q, S.query_start, S.block_table, S.seq_lens, S.mask, S.out)
        return S.out
    if op == "tables":
        return _plain_tables(S)
    if op == "accept":
        return _plain_accept(S)
    if op == "compact":
        return _plain_compact(S)
    return _plain_attention(S)


def _pools(S, lens):
    """Both pools' 16-bit patterns, and the lengths."""
    local = S.pool[:S.n_local].view(torch.int16)
    local.owner = S                          # the pools live as long as their handle
    return [local] + ([S.far[:S.n_far].view(torch.int16)] if S.n_far else []) + [lens]


def _padded(S):
    """Row of node i of request b (clamped), and whether there is one: [B][most]."""
    starts = S.query_start.long()
    i = torch.arange(S.most, device="cuda")
    live = i < (starts[1:] - starts[:-1])[:, None]
    return (starts[:-1, None] + i).clamp(max=S.T - 1), live


def _ancestors(S, rows, live):
    """[B][most][most]: node j is node i or above it. By doubling the way up."""
    none = S.most
    up = torch.where(live, S.parents.long()[rows], none)
    up = torch.where(up < 0, none, up)
    up = torch.cat([up, torch.full((S.B, 1), none, device="cuda")], 1)
    r = torch.eye(none + 1, dtype=torch.bool, device="cuda")[:, :none].repeat(S.B, 1, 1)
    for _ in range((S.most - 1).bit_length()):
        r |= r.gather(1, up[:, :, None].expand(-1, -1, none))
        up = up.gather(1, up)
    return r[:, :none]


def _plain_tables(S):
    rows, live = _padded(S)
    r = _ancestors(S, rows, live)
    starts = S.query_start.long()
    base = S.seq_lens.long() - (starts[1:] - starts[:-1])
    bit = torch.ones((), dtype=torch.int64, device="cuda") << torch.arange(64, device="cuda")
    wide = torch.zeros((S.B, S.most, S.words * 64), dtype=torch.int64, device="cuda")
    wide[:, :, :S.most] = r
    mask = (wide.view(S.B, S.most, S.words, 64) * bit).sum(-1)
    pos = base[:, None] + r.sum(-1) - 1
    return [mask[live], pos[live].to(torch.int32), base.to(torch.int32)]


def _plain_accept(S):
    rows, live = _padded(S)
    r = _ancestors(S, rows, live)
    parent, drafted, choice = (x.long()[rows] for x in (S.parents, S.drafted, S.choice))
    want = choice.gather(1, parent.clamp(min=0))
    i = torch.arange(S.most, device="cuda")
    if S.root_choice is not None:
        ok = drafted == torch.where(parent < 0, S.root_choice.long()[:, None], want)
    else:                                    # the first node is the last sampled token
        ok = (i == 0) | ((parent >= 0) & (drafted == want))
    ok &= live
    # of the confirmed children of a node the lowest
    at = torch.where(ok, parent + 1, S.most + 1)
    lowest = torch.full((S.B, S.most + 2), S.most, device="cuda").scatter_reduce(
        1, at, i.expand(S.B, -1), "amin")
    ok &= lowest.gather(1, at) == i
    taken = live & ~(r & ~ok[:, None, :]).any(-1)
    taken &= taken.cumsum(1) <= S.case["cap"]
    n = taken.sum(1)
    path = torch.where(taken, i, S.most).sort(1)[0][:, :S.case["cap"]]
    last = torch.where(taken, i, -1).amax(1)
    first = S.root_choice.long() if S.root_choice is not None else torch.full_like(n, -1)
    follow = torch.where(last < 0, first, choice.gather(1, last.clamp(min=0)[:, None])[:, 0])
    i32 = torch.int32
    return [torch.where(path == S.most, -1, path).to(i32), n.to(i32), follow.to(i32)]


def _parts(S, pool, far):
    """A pool's K and V as [block][token][head][channel] views of its patterns."""
    nhd = far and S.case["layout"] == "nhd"
    e = pool.view(torch.int16).view(pool.shape[0], 2, S.H * S.bs * D)
    if nhd:
        return [e[:, h].unflatten(1, (S.bs, S.H, D)) for h in (0, 1)]
    return [e[:, 0].unflatten(1, (S.H, S.bs, D)).transpose(1, 2),
            e[:, 1].unflatten(1, (S.H, D, S.bs)).permute(0, 3, 1, 2)]


def _plain_compact(S):
    """Every kept token of all layers read, then written to its place."""
    k = torch.arange(S.keep.shape[1], device="cuda")
    b, k = (k < S.n_keep[:, None]).nonzero(as_tuple=True)
    src, dst = S.base.long()[b] + S.keep.long()[b, k], S.base.long()[b] + k
    u, v = S.table[:, b, src // S.bs].long(), S.table[:, b, dst // S.bs].long()
    pools = [(S.pool, 0, S.n_local, False)] + ([(S.far, S.n_local, S.n_far, True)] if S.n_far else [])
    value = [None, None]
    for pool, first, n, far in pools:        # reads of both pools come before any write
        ids = torch.where((u >= first) & (u < first + n), u - first, n)
        for half, e in enumerate(_parts(S, pool, far)):
            x = e[ids, src % S.bs]
            value[half] = x if value[half] is None else torch.where(
                (u < first)[..., None, None], value[half], x)
    for pool, first, n, far in pools:
        ids = torch.where((v >= first) & (v < first + n), v - first, n)
        for half, e in enumerate(_parts(S, pool, far)):
            e[ids, (dst % S.bs).expand_as(ids)] = value[half]
    return _pools(S, (S.base + S.n_keep).to(torch.int32))


def _softmax(s, mask):
    """Weights over the last axis; zero for a row whose mask leaves nothing."""
    s = s.masked_fill_(~mask, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp_(s.sub_(torch.where(m == -math.inf, 0.0, m)))
    return p.div_(p.sum(-1, keepdim=True).clamp_min_(1e-30))


def _plain_attention(S):
    """Sequences padded to the longest, products and softmax in 32 bits."""
    B, H, N, most = S.B, S.H, S.width * S.bs, S.most
    ids = S.block_table.long().clamp(min=0)
    e = S.pool.view(S.dt).view(S.pool.shape[0], 2, H * S.bs * D)
    K = e[:, 0].unflatten(1, (H, S.bs, D))[ids].float().permute(0, 2, 1, 3, 4).reshape(B, H, N, D)
    V = e[:, 1].unflatten(1, (H, D, S.bs))[ids].float().permute(0, 2, 1, 4, 3).reshape(B, H, N, D)
    rows, live = _padded(S)
    G = S.Hq // H
    q = S.q.float()[rows] * (1.0 / math.sqrt(D))                       # [B][most][Hq][D]
    q = q.view(B, most, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * most, D)
    starts = S.query_start.long()
    base = S.seq_lens.long() - (starts[1:] - starts[:-1])
    t = torch.arange(N, device="cuda")
    node = (t - base[:, None])[:, None]                                 # [B][1][N]
    word = S.mask[rows].gather(2, (node.clamp(0, most - 1) >> 6).expand(B, most, N))
    mask = (node < 0) | ((node < most) & ((word >> (node & 63)) & 1 == 1))
    mask &= (t < S.seq_lens[:, None])[:, None]
    mask = mask[:, None, None].expand(B, 1, G, most, N).reshape(B, 1, G * most, N)
    o = _softmax(q @ K.transpose(-1, -2), mask) @ V
    o = o.view(B, H, G, most, D).permute(0, 3, 1, 2, 4).reshape(B, most, S.Hq, D)
    return o[live].to(S.out.dtype)


# ---- from the definition, in 64 bits --------------------------------------------------

def exact(case, seed):
    if case["op"] != "tree":                 # whole numbers and moved patterns
        return None
    S = _State()
    g = _inputs(case, seed, S)
    S.pool = torch.empty((S.nb, _block_bytes(case)), dtype=torch.uint8, device="cuda")
    _fill(g, S.pool, S.nb, S.dt)
    elems = S.pool.view(S.dt).double().view(S.nb, 2, -1)
    bs, H, G = S.bs, S.H, S.Hq // S.H
    table, parents = S.block_table.cpu().numpy(), S.parents.cpu().numpy()
    out = torch.zeros((S.T, S.Hq, D), dtype=torch.float64, device="cuda")
    row = 0
    for b, (ctx, n) in enumerate(S.pairs):
        N = ctx + n
        e = elems[_gpu(table[b, :-(-N // bs)].astype(np.int64))]
        K = e[:, 0].reshape(-1, H, bs, D).transpose(0, 1).reshape(H, -1, D)[:, :N]
        V = e[:, 1].reshape(-1, H, D, bs).permute(1, 0, 3, 2).reshape(H, -1, D)[:, :N]
        seen = np.zeros((n, N), dtype=bool)
        seen[:, :ctx] = True
        for i in range(n):                   # up to the root, step by step
            j = i
            while j >= 0:
                seen[i, ctx + j] = True
                j = parents[row + j]
        hidden = ~_gpu(seen)
        for head in range(S.Hq):
            s = S.q[row:row + n, head].double() @ K[head // G].T / math.sqrt(D)
            out[row:row + n, head] = torch.softmax(s.masked_fill(hidden, -math.inf), 1) @ V[head // G]
        row += n
    return out
