"""Refusals of the receiver's side at the edges of 64 bits, on a host without a GPU."""
import ctypes

import pytest

from test_cache_cpu import FAKE, L, cb, rows  # noqa: F401  (cb: the fixture)


@pytest.mark.parametrize("size", [(2**20, 2**20, 2**29), (2**20, 2**20, 2**24), (2**31 - 1, 2**31 - 1, 4), (2**16, 2**24, 2),
                                  (2**10, 2**30, 2**29), (0, 2**31 - 1, 2**29)])
def test_rotary_refuses_more_rows_than_64_bits_count(cb, size):
    """Row counts whose product is a multiple of 2^64, or negative in 64 bits, or just past 2^40."""
    assert cb._lib.cb_rotary(L(rows(cb, size=size)), 1, 8, FAKE, 8, 1.0, 0, 0, 1, None) == -2


def test_rotary_takes_no_rows_of_many(cb):
    """Nothing to do, with an axis of any length beside the empty one."""
    assert cb._lib.cb_rotary(L(rows(cb, size=(0, 2**20, 2**20))), 1, 8, FAKE, 8, 1.0, 0, 0, 1, None) == 0
