"""Window attention on the GPU against the definition in 64 bits."""
import pytest
import torch

import window_harness as wh
from window_harness import FULL, Case

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 8, 2, 64), ("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("bf16", 6, 3, 96), ("bf16", 8, 8, 40), ("bf16", 4, 1, 256),
          ("bf16", 32, 8, 128), ("bf16", 6, 2, 200), ("f32", 8, 2, 64), ("f32", 6, 3, 40), ("f32", 5, 1, 128), ("f32", 4, 2, 256), ("f32", 4, 2, 96)]
LENS = [[(0, 1)], [(0, 5)], [(15, 1)], [(16, 1)], [(17, 3), (0, 0), (40, 0), (0, 2)], [(100, 1), (0, 33), (257, 70), (31, 2)], [(433, 130)]]
WINDOWS = [(1, 0), (5, 3), (33, 40), (64, 4), (300, 17), (FULL, 0), (70, FULL)]


def run_and_check(c, window, n_first, weight_step=2.0 ** -8):
    print(f"[case] {c.dtype} {c.hq}/{c.hkv} D={c.dim} {c.lens} window={window} first={n_first}", flush=True)
    got = c.run(window, n_first)
    wh.check_pool(c, got)
    for l in range(c.layers):
        wh.check_attn(c, got, window, n_first, l, weight_step if c.dtype == "bf16" and c.dim == 128 else 0.0)


@pytest.mark.parametrize("dtype,hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("window,n_first", WINDOWS)
def test_lengths(dtype, hq, hkv, dim, window, n_first):
    for i, lens in enumerate(LENS):
        run_and_check(Case(lens, hq, hkv, dim, dtype, seed=100 + i), window, n_first)


@pytest.mark.parametrize("dtype,hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("pieces", ["2", "7"])
@pytest.mark.parametrize("tile", ["1", "2"])
def test_cut_tiles(dtype, hq, hkv, dim, pieces, tile, monkeypatch):
    monkeypatch.setenv("CALVO_ATTN_SPLITS", pieces)
    monkeypatch.setenv("CALVO_ROWS_TILE", tile)
    for window, n_first in [(5, 3), (64, 100), (300, 17), (FULL, 0)]:
        run_and_check(Case([(100, 1), (0, 33), (257, 70)], hq, hkv, dim, dtype, seed=7), window, n_first)


@pytest.mark.parametrize("dim", [64, 128])
def test_long_context(dim):
    run_and_check(Case([(6007, 1), (3001, 40), (20011, 2)], 8, 2, dim, seed=3), 2500, 100)
    run_and_check(Case([(6007, 1)], 16, 2, dim, seed=4, layers=2), FULL, 0)


# CALVO_ATTN_VARIANT: 64 or 32 query rows per wave in the pipelined kernels, 5 the packed rows
@pytest.mark.parametrize("variant", ["3", "4", "5"])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (32, 8), (5, 1), (4, 2)])
@pytest.mark.parametrize("pieces", ["0", "2", "7"])
def test_kernels_of_128_wide_heads(variant, hq, hkv, pieces, monkeypatch):
    monkeypatch.setenv("CALVO_ATTN_VARIANT", variant)
    if pieces != "0":
        monkeypatch.setenv("CALVO_ATTN_SPLITS", pieces)
    for window, n_first in WINDOWS:
        for i, lens in enumerate([[(0, 1), (17, 3)], [(100, 1), (0, 33), (257, 70), (31, 2)], [(433, 130), (1200, 65)]]):
            run_and_check(Case(lens, hq, hkv, 128, seed=300 + i), window, n_first)


@pytest.mark.parametrize("variant", ["3", "4", "5"])
def test_long_contexts_of_128_wide_heads(variant, monkeypatch):
    """The steady loop with and without whole sub-tiles of first tokens in front."""
    monkeypatch.setenv("CALVO_ATTN_VARIANT", variant)
    for window, n_first in [(1000, 0), (1300, 300), (777, 1), (FULL, 0)]:
        run_and_check(Case([(6007, 40), (2048, 2)], 8, 2, 128, seed=31), window, n_first)


def test_scale():
    c = Case([(50, 20)], seed=5)
    wh.check_attn(c, c.run(30, 2, scale=0.5), 30, 2, scale=0.5)


@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 128), ("bf16", 6, 2, 64), ("bf16", 4, 1, 256), ("f32", 6, 3, 64), ("f32", 4, 2, 128)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("pieces", ["0", "3"])
@pytest.mark.parametrize("variant", ["3", "4", "5"])
def test_hidden_keys_do_not_reach_a_row(dtype, hq, hkv, dim, value, pieces, variant, monkeypatch):
    """K and V of cached tokens and of new ones hold `value`: rows that do not see them are within the bounds of a pool without.  (Not its
    bits: how far a row's softmax reference lies above its maximum depends on the rows beside it.)"""
    if variant != "5" and (dtype, dim) != ("bf16", 128):
        pytest.skip("one kernel only")
    monkeypatch.setenv("CALVO_ATTN_SPLITS", pieces)
    monkeypatch.setenv("CALVO_ATTN_VARIANT", variant)
    c = Case([(150, 90)], hq, hkv, dim, dtype, seed=11)
    window, n_first, poisoned = 40, 5, [3, 30, 120, 149, 150 + 20, 150 + 61]
    t = c.tables[0]
    clean = c.pool[0, t[0], :, 3].clone()
    for p in poisoned:
        if p < 150:
            c.pool[0, t[p // 16], :, p % 16] = value
        else:
            c.k[0, p - 150] = value
            c.v[0, p - 150] = value
    got = c.run(window, n_first)
    seen = wh.wo.sees(range(150, 240), poisoned, window, n_first)
    apart = ~seen[:, 1:].any(axis=1)                          # position 3 is among the first tokens: every row sees it
    c.pool[0, t[0], :, 3] = clean
    alone = c.run(window, n_first)
    assert apart.any() and not apart.all()
    wh.check_attn(c, alone, window, n_first, weight_step=2.0 ** -8 if dtype == "bf16" and dim == 128 else 0.0, rows=apart)
    assert not torch.isfinite(alone["out"][0, ~apart].float()).all(dim=-1).any()
    assert not torch.isfinite(got["out"][0].float()).all(dim=-1).any()
