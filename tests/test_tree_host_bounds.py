"""Refusals of the operators of include/ema_tree.h on the host: starts at the ends of their
type."""
import numpy as np
import pytest

from test_tree_host import _Mask, host, i32, pytestmark, refused, z  # noqa: F401

LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("starts", [[0, 2, LOW], [0, HIGH, LOW], [0, LOW, 2], [0, HIGH, 2], [0, 1, HIGH],
                                    [LOW, 0, 2]])
def test_starts_at_the_ends_of_their_type(host, starts):
    ema, h = host
    for message in (
            refused(ema, ema.tree_tables, h, z(2) - 1, i32(starts), i32([HIGH, HIGH]), _Mask(2, 1)),
            refused(ema, ema.tree_accept, h, z(2) - 1, i32(starts), z(2), z(2), z(2, 3), z(2), z(2))):
        assert "query_start" in message
