"""Limits of the calls around a 4-bit cache, on both sides, as far as the host decides them."""

import pytest

from tests.test_operators_host import _refused, _tables


@pytest.mark.parametrize("entries", ["page_indices_len", "free_pages_len"])
def test_step_tables_sum_in_32_bits(entries):
    """A round of 1024 requests moves and lists up to 2^30 pages, which the kernel adds to a number of entries in 32 bits: 2^30 entries would be one too many."""
    for n in (1 << 30, (1 << 31) - 1):
        _refused(_tables(**{entries: n}), 2, "2^30")
    # one fewer is taken: the next check has its turn
    _refused(_tables(**{entries: (1 << 30) - 1, "kv_len": None}), 1, "NULL")
