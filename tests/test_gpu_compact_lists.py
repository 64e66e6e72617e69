"""Compaction of long lists with what is out of range in them: entries that do not ascend or
lie past the table, bases and counts, table entries outside both pools under sources and
places, in full chunks of a list and in those that its pieces cut short. Pools byte for
byte, the count exact."""
import numpy as np
import pytest
import torch

from ops_harness import i32
from oracle import trees
from test_gpu_tree import D, Pools, full

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ema():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_27040_amd import ema as m
    return m


def expect(p, table, base, keep, n_keep):
    """The pools and the count of what include/ema_tree.h says of such lists."""
    L, B, width = table.shape
    cap, blocks, errors = keep.shape[1], p.n_local + p.n_far, 0
    room = width * p.bs
    for b in range(B):
        n = min(max(n_keep[b], 0), cap)
        errors += int(n != n_keep[b]) + int(base[b] < 0)
        if base[b] < 0:
            continue
        for k in range(n):
            src = int(keep[b, k])
            before = int(keep[b, k - 1]) if k else -1
            if src < k or src <= before or base[b] + src >= room:
                errors += 1
                continue
            if src == k:
                continue
            for l in range(L):
                ids = [table[l, b, (base[b] + t) // p.bs] for t in (src, k)]
                if any(i < 0 or i >= blocks for i in ids):
                    errors += 1
                    continue
                trees.kv_compact(*p.host, p.nhd, p.table[l:l + 1, b:b + 1], [base[b] + k], [[src - k]],
                                 [1], p.H, D, p.bs)
    return errors


def run(ema, p, table, base, keep, n_keep):
    new = full((len(base),))
    errors = expect(p, table, base, keep, n_keep)
    ema.kv_compact(p.h, i32(table), i32(base), i32(keep), i32(n_keep), new_lens=new)
    p.same()
    assert ema.slice_device_errors(p.h) == errors
    n = np.clip(n_keep, 0, keep.shape[1])
    assert np.array_equal(new.cpu().numpy(), (np.asarray(base, np.int64) + n).astype(np.int32))
    return errors


def spread(rng, n, of):
    """n ascending tokens of `of`."""
    return np.sort(rng.permutation(of)[:n])


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("bs,dense", [(16, True), (16, False), (64, False), (256, True)])
def test_bad_table_entries(ema, bs, dense, layout):
    """Some under sources only, some under places. dense: chunks of 64 places; else every 9th
    token is kept, and 24 pieces end a chunk."""
    p = Pools(ema, 2, [1900, 700, 1900], 2, bs, layout, 0.4, seed=bs + dense)
    try:
        rng = p.rng
        base = np.array([3, 0, 1])
        n = [1100, 400, 1000] if dense else [200, 75, 190]
        keep = np.full((3, max(n) + 3), -9)
        for b, of in enumerate([1890, 700, 1899]):
            keep[b, :n[b]] = spread(rng, n[b], of) if dense else \
                np.arange(n[b]) * 9 + rng.integers(0, 9, n[b])
        table = p.table.copy()
        last = [-(-x // bs) for x in (1900, 700, 1900)]
        # first, middle and last blocks: under the first and later chunks, of places and of sources
        table[0, 0, 0] = -1
        table[1, 0, last[0] // 2] = p.n_local + p.n_far
        table[1, 2, last[2] - 1] = 2 ** 31 - 1
        table[0, 1, last[1] // 2] = -2 ** 31
        if bs == 16:
            for l, b, j in ((0, 2, 5), (0, 2, 9), (1, 2, 40), (1, 1, 12)):
                table[l, b, j] = -7
        assert run(ema, p, table, base, keep, n) > 10       # the inputs have some
    finally:
        p.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_lists_that_do_not_ascend_or_end(ema, layout):
    lens = [1000] * 8
    p = Pools(ema, 2, lens, 1, 16, layout, 0.5, seed=7)
    try:
        rng = p.rng
        room = p.table.shape[2] * 16
        keep = np.stack([spread(rng, 300, 700) for _ in range(8)])
        keep[0, [0, 70, 71, 150]] = [-1, 3, 3, -2 ** 31]             # below, twice, far below
        keep[1, 290:] = room + np.arange(10)                         # past the table
        keep[1, 299] = 2 ** 31 - 1
        keep[2, 100:110] = keep[2, 110:120]                          # up, then down again
        keep[3] = np.arange(300)                                     # nothing moves
        keep[3, 64:66] = 0                                           # ... of 298
        keep[4, :] = -5                                              # nothing at all
        base = np.array([0, 5, 17, 3, 0, -1, room + 5, 2 ** 31 - 1])
        n = [300, 300, 299, 300, 300, 300, 12, 5]
        run(ema, p, p.table, base, keep, n)
    finally:
        p.close()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("cap", [9, 10, 80])
def test_counts_out_of_range(ema, cap, layout):
    p = Pools(ema, 1, [200] * 6, 2, 16, layout, 0.5, seed=cap)
    try:
        keep = np.stack([spread(p.rng, cap, 180) for _ in range(6)])
        n = [cap, cap + 1, -1, 2 ** 31 - 1, -2 ** 31, 0]
        run(ema, p, p.table, np.array([0, 3, 7, 1, 0, 20]), keep, n)
    finally:
        p.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_short_lists_in_wide_arrays(ema, layout):
    """As a path has them whose capacity is the tree's nodes: the same as in narrow ones."""
    rng = np.random.default_rng(5)
    n = [0, 1, 3, 9, 12, 4]
    lists = [spread(rng, x, 16) for x in n]
    after = []
    for cap in (12, 16, 64, 1000):
        p = Pools(ema, 3, [60] * 6, 8, 16, layout, 0.3, seed=6)
        try:
            keep = np.full((6, cap), -1)
            for b, x in enumerate(lists):
                keep[b, :n[b]] = x
            assert run(ema, p, p.table, np.array([40, 44, 0, 15, 17, 31]), keep, n) == 0
            after.append([x.copy() for x in p.host])
        finally:
            p.close()
    assert all(np.array_equal(a, b) for x in after for a, b in zip(x, after[0]))
