"""Plans over 8-bit pools: what is cut, into how much, and which kernel takes it (no GPU needed)."""
import numpy as np
import pytest

from paper_2603_21257_amd import binding as cb

FULL = 2 ** 31 - 1
ROWS = -1


def plan(lens, hq, hkv, dim, window=FULL):
    reqs, at = [], 0
    for c, n in lens:
        m = -(-(c + n) // 16)
        reqs.append(cb.make_window_request(np.arange(at, at + m), c, n, -1))
        at += m
    kernel, runs = cb.calvo_window_plan(hq, hkv, dim, cb.CALVO_E4M3, at, 256, reqs, window, 0)
    return kernel, np.asarray(runs)


@pytest.mark.parametrize("hq,hkv,dim", [(32, 8, 128), (64, 8, 64), (8, 8, 96), (32, 8, 256)])
def test_one_long_request_among_many_short_ones(hq, hkv, dim):
    """Its pieces do not get longer with the number of the others, and no piece is a third of it."""
    for others in (3, 23, 40):
        lens = [(60000, 1)] + [(50 + 7 * i, 1) for i in range(others)]
        kernel, runs = plan(lens, hq, hkv, dim)
        assert kernel == ROWS
        mine = runs[runs[:, 0] == 0]
        assert 8 <= mine[0, 6] <= 32
        assert (mine[:, 4] - mine[:, 3]).max() * 32 <= 60000 / 6
        assert len(runs) * hkv <= 4 * 256


def test_even_batches_fill_the_chip_once():
    _, runs = plan([(4096, 1)] * 4, 32, 8, 128)
    assert 128 <= len(runs) * 8 <= 512


def test_small_launches_stay_on_packed_rows():
    assert plan([(45, 1), (0, 1015)], 8, 8, 128)[0] == ROWS
    assert plan([(1543, 435)], 6, 3, 128, 4097)[0] == ROWS
    assert plan([(16384, 2048)], 32, 8, 128)[0] != ROWS
