"""What an append leaves in an 8-bit pool, byte by byte, wherever the definition says exactly what that is: V, and K that is not rotated."""
import numpy as np
import pytest
import torch

from e4m3_harness import Case8, inv_freq
from oracle import e4m3_oracle as eo
from window_harness import FULL

pytestmark = pytest.mark.gpu
B = 16


def check_bytes(c, got, k_exact=True):
    """Nearest values, ties to the even one; a tile whose scale is NaN holds zeros.  Of a zero the sign is free."""
    tiles = 0
    for l in range(c.layers):
        gk, gv, gs = eo.parts(got["pool"][l], c.hkv, c.dim)
        ok, ov, osc = eo.parts(c.pool[l], c.hkv, c.dim)
        new = c.k[l].double().numpy(), c.v[l].double().numpy()
        for r, ((cached, n), t) in enumerate(zip(c.lens, c.tables)):
            for b in range(cached // B, -(-(cached + n) // B) if n else 0):
                lo, hi, s = max(cached, b * B), min(cached + n, b * B + B), t[b]
                a, e = lo - b * B, hi - b * B
                for h in range(c.hkv):
                    for which in (0, 1) if k_exact else (1,):
                        x = new[which][c.cu[r] + lo - cached:c.cu[r] + hi - cached, h]
                        held, old = (gk[s, h], ok[s, h]) if which == 0 else (gv[s, h].T, ov[s, h].T)
                        before, now, scale = eo.append_block(old, osc[s, which, h], a, x)
                        name = f"layer {l} request {r} block {b} head {h} {'KV'[which]}"
                        want = np.zeros((B, c.dim), np.uint8)
                        if np.isnan(scale):
                            assert np.isnan(gs[s, which, h]), name
                        else:
                            assert gs[s, which, h] == scale, name
                            want[:a], want[a:e] = before, eo.encode(now)
                        zero = ((held | want) & 127) == 0
                        assert ((held == want) | zero).all(), (name, np.argwhere((held != want) & ~zero)[:3].tolist())
                        tiles += 1
    assert tiles


@pytest.mark.parametrize("hq,hkv,dim", [(8, 2, 64), (8, 2, 128), (6, 3, 96), (4, 4, 48), (4, 1, 256), (6, 2, 208), (2, 2, 16)])
def test_nearest_values(hq, hkv, dim):
    for i, lens in enumerate([[(0, 1)], [(31, 3), (0, 0), (40, 0), (0, 2)], [(100, 1), (0, 33), (257, 70), (5, 11)], [(0, 16), (47, 1)]]):
        c = Case8(lens, hq, hkv, dim, seed=90 + i, layers=2)
        check_bytes(c, c.run(FULL))
        check_bytes(c, c.run(FULL, rope=(inv_freq(dim), dim, bool(i % 2))), k_exact=False)


def test_ties_and_the_lower_end():
    """Every significand of bf16 at exponents from the scale's largest value to below its least one."""
    c = Case8([(0, 16), (7, 9)], 2, 2, 128, seed=4)
    m = (1 + torch.arange(128).double() / 128)
    for x in (c.k, c.v):
        for i in range(c.total):
            x[0, i, 0] = m * 2.0 ** (-i)
            x[0, i, 1] = -m * 2.0 ** (i - 30)
        x[0, 0, :, 0] = x[0, 16, :, 0] = 1.75
    check_bytes(c, c.run(FULL))


@pytest.mark.parametrize("size", [-100.0, -20.0, -3.0, 3.0, 20.0])
def test_scales_that_grow_and_stay(size):
    c = Case8([(3, 1), (9, 5), (15, 20), (0, 4)], 4, 2, 64, seed=9, size=size)
    check_bytes(c, c.run(FULL))


@pytest.mark.parametrize("dim", [48, 64, 128, 256])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_tiles_without_a_finite_scale_hold_zeros(dim, value):
    c = Case8([(20, 3), (0, 5), (40, 30)], 4, 2, dim, seed=3)
    c.k[0, 1, 0, 7] = value
    c.v[0, 4, 1, dim - 1] = value
    c.k[0, 30, 1, 0] = value
    check_bytes(c, c.run(FULL))
    # a block that has such a scale already keeps it
    c = Case8([(20, 3)], 4, 2, dim, seed=3)
    n8 = 2 * 16 * dim
    c.pool[0, c.tables[0][1], 2 * n8:2 * n8 + 16] = np.float32([np.inf, 1.0, np.nan, 2.0 ** -6]).view(np.uint8)
    check_bytes(c, c.run(FULL))
