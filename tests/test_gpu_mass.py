"""Gathered attention weights on the GPU against the definition in 64 bits."""
import pytest
import torch

import window_harness as wh
from window_harness import FULL, Case

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 8, 2, 64), ("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("bf16", 6, 3, 96), ("bf16", 8, 8, 40), ("bf16", 4, 1, 256),
          ("bf16", 32, 8, 128), ("f32", 8, 2, 64), ("f32", 6, 3, 40), ("f32", 5, 1, 128), ("f32", 4, 2, 256)]


def given(c, seed=9):
    return torch.rand((c.layers, len(c.lens) + 1, c.hkv, c.stride()), generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype,hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("window,n_first", [(1, 0), (5, 3), (33, 40), (300, 17), (FULL, 0)])
def test_lengths(dtype, hq, hkv, dim, window, n_first):
    for i, lens in enumerate([[(0, 1)], [(0, 5)], [(16, 1)], [(17, 3), (0, 0), (40, 0), (0, 2)], [(100, 1), (0, 33), (257, 70), (31, 2)], [(433, 130)]]):
        c = Case(lens, hq, hkv, dim, dtype, seed=200 + i)
        print(f"[case] {dtype} {hq}/{hkv} D={dim} {lens} window={window} first={n_first}", flush=True)
        wh.check_mass(c, c.run(window, n_first, mass=True), window, n_first)
        for last_rows in (0, 1, 20):
            m = given(c)
            wh.check_mass(c, c.run(window, n_first, mass=True, last_rows=last_rows, mass_in=m), window, n_first, last_rows, m)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_in_place_and_layers(dtype, dim):
    c = Case([(300, 20), (64, 1)], 8, 2, dim, dtype, seed=5, layers=2)
    m = given(c)
    got = c.run(100, 4, mass=True, mass_in=m, in_place=True)
    for l in range(2):
        wh.check_mass(c, got, 100, 4, 0, m, l, left=None)


def test_long_and_same_bits():
    c = Case([(5003, 300), (9000, 1)], 8, 2, 128, seed=6)
    first = c.run(FULL, 0, mass=True)
    wh.check_mass(c, first, FULL, 0)
    assert torch.equal(first["mass"], c.run(FULL, 0, mass=True)["mass"])


def test_rows_weigh_one_in_all():
    """The weights that a row gives away are its softmax: all of a batch's sums add up to the number of rows and heads."""
    c = Case([(0, 700)], 8, 2, 128, seed=8)
    total = c.run(150, 10, mass=True)["mass"][0, 0, :, :700].double().sum(dim=1)
    assert torch.allclose(total, torch.full_like(total, 700.0 * 4), rtol=1e-5, atol=0)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f32", 64)])
def test_hidden_keys(dtype, dim):
    """NaN in K of tokens that no counted row sees, and behind the last token: nothing of it in any weight."""
    c = Case([(150, 9)], 8, 2, dim, dtype, seed=12)
    t = c.tables[0]
    c.pool[0, t[1], :, 3] = float("nan")
    got = c.run(40, 5, mass=True)
    c.pool[0, t[1], :, 3] = 0.0
    wh.check_mass(c, got, 40, 5)
