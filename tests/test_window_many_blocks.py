"""Batches whose tables, one behind the other, have places past 32 bits (no GPU needed)."""
import numpy as np
import pytest

from paper_2603_21257_amd import binding as cb

BLOCKS = 1 << 20


def batch(n):
    """n requests over the same cached blocks, which none of them stores to."""
    table = np.arange(BLOCKS, dtype=np.int32)
    return [cb.make_window_request(table, 16 * BLOCKS, 0, -1) for _ in range(n)]


def plan(reqs):
    return cb.calvo_window_plan(8, 2, 64, cb.CALVO_BF16, BLOCKS, 256, reqs, 100, 0)


def test_places_in_the_tables_are_32_bits_wide():
    assert plan(batch(3))[1].shape == (0, 7)
    with pytest.raises(cb.CalvoError, match="too many tokens in the batch") as e:
        plan(batch(2048))
    assert e.value.code == cb.CALVO_EINVAL
