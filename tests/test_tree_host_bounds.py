"""Refusals of the operators of include/ema_tree.h on the host: starts at the ends of their
type, blocks named twice, outputs that overlap other arrays,
masks of another shape."""
import numpy as np
import pytest

from test_tree_host import _Mask, _Q, host, i32, pytestmark, refused, z  # noqa: F401

LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("starts", [[0, 2, LOW], [0, HIGH, LOW], [0, LOW, 2], [0, HIGH, 2], [0, 1, HIGH],
                                    [LOW, 0, 2]])
def test_starts_at_the_ends_of_their_type(host, starts):
    ema, h = host
    for message in (
            refused(ema, ema.tree_tables, h, z(2) - 1, i32(starts), i32([HIGH, HIGH]), _Mask(2, 1)),
            refused(ema, ema.tree_accept, h, z(2) - 1, i32(starts), z(2), z(2), z(2, 3), z(2), z(2))):
        assert "query_start" in message


def test_a_block_named_twice_is_refused(host):
    ema, h = host

    def f(table, base, keep, n):
        ema.kv_compact(h, i32(table), i32(base), i32(keep), i32(n))

    two = [[0, 17, 18, -1], [1, 20, 47, -1]]
    f([[[0, 1, -1], [13, 3, 17]]], [0, 0], two, [3, 3])
    f([[[0, 1, 5], [13, 3, 5]]], [0, 0], two, [3, 0])                  # no token of the second request
    f([[[0, 1, 5], [0, 1, 5]]], [0, 0], [[0, 1, 2], [1, 2, 4]], [3, 3])    # nor of the first
    f([[[0, 1, 4], [13, 3, 4]]], [0, 0], [[0, 17, 18], [1, 2, 31]], [3, 3])  # not moved there
    bad = [([[[0, 0, -1], [13, 3, 17]]], [3, 3]),                      # of one request
           ([[[0, 1, -1], [13, 3, 1]]], [3, 3]),                       # of two
           ([[[0, 1, -1], [13, 3, 17]], [[2, 4, -1], [14, 0, 16]]], [3, 3])]     # of two layers
    for table, n in bad:
        assert "twice" in refused(ema, f, table, [0, 0], two, n)
    f([[[0, 1, -1], [13, 3, 17]], [[2, 4, -1], [14, 5, 16]]], [0, 0], two, [3, 3])


def test_outputs_that_overlap_are_refused(host):
    ema, h = host
    starts, lens = i32([0, 2, 5]), i32([9, 9])

    def tables(parents=z(5) - 1, seq_lens=lens, **out):
        ema.tree_tables(h, parents, starts, seq_lens, _Mask(5, 1), **out)

    p, both = z(5) - 1, z(7)
    tables(p, positions=z(5), base=z(2))
    tables(p, positions=both[:5], base=both[5:])                       # side by side
    for out in (dict(base=lens), dict(base=starts[1:]), dict(positions=p), dict(base=p[3:]),
                dict(positions=both[:5], base=both[4:6])):
        assert "overlaps" in refused(ema, tables, p, **out)

    def accept(path=None, n_path=None, next_token=None, root=None):
        ema.tree_accept(h, p, starts, p, p, z(2, 3) if path is None else path,
                        z(2) if n_path is None else n_path, z(2) if next_token is None else next_token,
                        root_choice=root)

    wide, two = z(10), z(2)
    accept(wide[:6].reshape(2, 3), wide[6:8], wide[8:])
    for a in (dict(path=wide[:6].reshape(2, 3), n_path=wide[5:7]), dict(n_path=two, next_token=two),
              dict(next_token=two, root=two), dict(n_path=p[:2]), dict(next_token=starts[:2])):
        assert "overlaps" in refused(ema, accept, **a)

    table, keep = i32([[[0, 1], [2, 3]]]), i32([[1, 5], [0, 3]])
    base, n = i32([0, 3]), i32([2, 2])
    ema.kv_compact(h, table, base, keep, n, new_lens=z(2))
    for out in (base, n, keep[1], table[0, 0]):
        assert "overlaps" in refused(ema, ema.kv_compact, h, table, base, keep, n, new_lens=out)


def test_masks_of_another_shape(host):
    ema, h = host
    f = lambda mask: ema.paged_tree_attention(h, _Q(8, 4), i32([0, 8]), i32([[0, 1]]), i32([20]), mask,
                                              None)
    f(_Mask(8, 1))
    for shape in ((), (8,), (7, 1), (9, 1), (8, 1, 1)):
        assert "mask" in refused(ema, f, _Mask(*shape))
