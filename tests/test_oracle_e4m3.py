"""Pins of the 8-bit oracle: the number format, the rotation, and the planning of launches over such pools; no GPU."""
import numpy as np
import pytest
import torch

from oracle import e4m3_oracle as eo
from paper_2603_21257_amd import binding as cb
from window_harness import FULL


def test_bytes_are_the_ocp_format():
    b = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(b).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(eo.decode(b), want, equal_nan=True)
    assert eo.VALUES[126] == 448 and eo.VALUES[1] == 2.0 ** -9
    finite = b[np.isfinite(want)]
    assert np.array_equal(eo.encode(eo.decode(finite)), finite)
    x = np.concatenate([np.random.default_rng(1).uniform(-448, 448, 4000), (eo.VALUES[:126] + eo.VALUES[1:127]) / 2, [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -11]])
    assert np.array_equal(eo.encode(x), torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_least_scale():
    for e in (-40, -3, 0, 7):
        assert eo.least_scale(448 * 2.0 ** e) == 2.0 ** e
        assert eo.least_scale(448.0001 * 2.0 ** e) == 2.0 ** (e + 1)
        assert eo.least_scale(225 * 2.0 ** e) == 2.0 ** e
        assert eo.least_scale(224 * 2.0 ** e) == 2.0 ** (e - 1)
    assert eo.least_scale(0.0) == 2.0 ** -126


def test_rotation_keeps_lengths_and_composes():
    x = np.random.default_rng(2).standard_normal((5, 3, 16))
    f = np.float32([1, 0.1, 0.01, 0.001])
    for inter in (False, True):
        a = eo.rotate(x, np.arange(5), f, 8, inter)
        assert np.allclose((a ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(a[..., 8:], x[..., 8:])
        assert np.allclose(eo.rotate(a, 7 - np.arange(5), f, 8, inter), eo.rotate(x, np.full(5, 7), f, 8, inter))
    # a quarter of a turn
    y = eo.rotate(np.float64([[[1, 2, 3, 4]]]), [1], [np.pi / 2, 0.0], 4, False)
    assert np.allclose(y, [[[-3, 2, 1, 4]]])
    y = eo.rotate(np.float64([[[1, 2, 3, 4]]]), [1], [np.pi / 2, 0.0], 4, True)
    assert np.allclose(y, [[[-2, 1, 3, 4]]])


def test_block_bytes():
    for hkv, dim in ((8, 128), (1, 16), (3, 96), (5, 256)):
        n = cb.calvo_block_bytes(hkv, dim, cb.CALVO_E4M3)
        assert n == eo.block_bytes(hkv, dim) and n % 128 == 0
        assert cb.calvo_block_bytes(hkv, dim, cb.CALVO_BF16) == 2 * 16 * hkv * dim * 2
        assert cb.calvo_block_bytes(hkv, dim, cb.CALVO_F32) == 2 * 16 * hkv * dim * 4
    for args in ((8, 40, cb.CALVO_E4M3), (8, 264, cb.CALVO_E4M3), (1 << 20, 256, cb.CALVO_E4M3), (8, 128, 3)):
        with pytest.raises(cb.CalvoError):
            cb.calvo_block_bytes(*args)


@pytest.mark.parametrize("hq,hkv,dim", [(8, 2, 64), (32, 8, 128), (5, 1, 128), (6, 3, 96), (4, 1, 256), (32, 1, 80)])
@pytest.mark.parametrize("window,n_first", [(1, 0), (5, 3), (64, 4), (300, 17), (4096, 64), (FULL, 0), (70, FULL)])
def test_plans_cover_what_rows_see(hq, hkv, dim, window, n_first):
    """Every (row, visible 32-key sub-tile) is met exactly once, and pieces marked as full hold no hidden key."""
    group = hq // hkv
    for lens in ([(0, 1)], [(100, 1), (0, 33), (257, 70)], [(6007, 1), (3001, 40)], [(40000, 1)], [(5000, 300)]):
        at, reqs = 0, []
        for c, n in lens:
            m = -(-(c + n) // 16)
            reqs.append(cb.make_window_request(np.arange(at, at + m), c, n, -1))
            at += m
        _, runs = cb.calvo_window_plan(hq, hkv, dim, cb.CALVO_E4M3, at, 256, reqs, window, n_first)
        for r, (c, n) in enumerate(lens):
            mine = runs[runs[:, 0] == r]
            for row in sorted({0, 1, n * group // 2, n * group - 1}):
                if not 0 <= row < n * group:
                    continue
                pos = c + row // group
                met = np.zeros((c + n) // 32 + 4, int)
                for _, r0, r1, s0, s1, full, _ in mine:
                    if r0 <= row < r1:
                        met[s0:s1] += 1
                        if full:
                            assert 32 * s1 - 1 <= pos and (32 * s0 > pos - window or 32 * s1 <= n_first)
                t = np.arange(pos + 1)
                seen = np.unique(t[(t > pos - window) | (t < n_first)] // 32)
                assert (met[seen] == 1).all() and met.max() == 1


def test_refusals_without_a_gpu():
    reqs = [cb.make_window_request([0, 1], 20, 4, -1)]
    with pytest.raises(cb.CalvoError, match="multiple of 16"):
        cb.calvo_window_plan(8, 2, 40, cb.CALVO_E4M3, 8, 256, reqs, FULL)
    with pytest.raises(cb.CalvoError, match="8-bit pool"):
        cb.calvo_evict_check(2, 64, cb.CALVO_E4M3, 8, [cb.make_evict_request([0], 8, [1], 4)], 1)
