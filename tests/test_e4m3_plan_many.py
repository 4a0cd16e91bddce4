"""Plans over 8-bit pools where the chip is full of short requests: the long one among them is cut all the same (no GPU needed)."""
import numpy as np
import pytest

from test_e4m3_plan import ROWS, plan

START = 20                                             # what a workgroup costs besides its 32-key sub-tiles, in those
CUS = 256


def longest_and_mean(others, hq, hkv, dim, long=60000):
    """Of a batch with one long request: its pieces, the longest one, and what a compute unit has to do on average, in sub-tiles."""
    kernel, runs = plan([(long, 1)] + [(50 + 7 * (i % 256), 1) for i in range(others)], hq, hkv, dim)
    assert kernel == ROWS
    mine, length = runs[runs[:, 0] == 0], runs[:, 4] - runs[:, 3]
    assert (runs[:, 6] > 1).sum() * hkv <= 4 * CUS       # what is merged stays bounded
    return mine[0, 6], length.max(), (length + START).sum() * hkv / CUS


@pytest.mark.parametrize("hq,hkv,dim", [(32, 8, 128), (64, 8, 64), (8, 8, 96), (32, 8, 256), (16, 2, 80)])
@pytest.mark.parametrize("others", [100, 126, 127, 128, 255, 400, 511, 600, 900])
def test_one_long_request(hq, hkv, dim, others):
    """No piece is longer than a sixth of it, or than twice the chip's work for everything: one order of the workgroups ends within mean + longest."""
    pieces, longest, mean = longest_and_mean(others, hq, hkv, dim)
    assert pieces <= 32
    assert longest <= max(60000 / 32 / 6, 2 * mean)


def test_pieces_do_not_fall_off_a_cliff():
    """One request more does not turn a cut launch into one that is not."""
    for others in range(90, 700, 7):
        pieces, longest, mean = longest_and_mean(others, 32, 8, 128)
        assert longest <= max(60000 / 32 / 6, 2 * mean), others


@pytest.mark.parametrize("n", [64, 128, 256, 600])
def test_even_batches_stay_whole(n):
    """Where every request is as long as the others and the chip is full, nothing is cut."""
    runs = plan([(4096, 1)] * n, 32, 8, 128)[1]
    assert len(runs) == n and np.all(runs[:, 6] == 1)
