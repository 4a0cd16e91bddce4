"""Attention over a pool of 8-bit floats on the GPU against the definition in 64 bits, on the blocks as the append left them."""
import numpy as np
import pytest
import torch

import e4m3_harness as eh
import window_harness as wh
from e4m3_harness import Case8
from oracle import e4m3_oracle as eo
from paper_2603_21257_amd import binding as cb
from window_harness import FULL

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

SHAPES = [(8, 2, 64), (8, 2, 128), (5, 1, 128), (6, 3, 96), (8, 8, 48), (4, 1, 256), (6, 2, 208), (32, 8, 128), (32, 1, 80), (2, 2, 16)]
LENS = [[(0, 1)], [(0, 5)], [(15, 1)], [(16, 1)], [(17, 3), (0, 0), (40, 0), (0, 2)], [(100, 1), (0, 33), (257, 70), (31, 2)], [(433, 130)],
        [(63, 1), (64, 1), (127, 2)]]
WINDOWS = [(1, 0), (5, 3), (33, 40), (64, 4), (300, 17), (FULL, 0), (70, FULL)]


def run_and_check(c, window, n_first, **kw):
    print(f"[case] {c.hq}/{c.hkv} D={c.dim} {c.lens} window={window} first={n_first}", flush=True)
    got = c.run(window, n_first, **kw)
    eh.check_append8(c, got)
    for l in range(c.layers):
        wh.check_attn(c, got, window, n_first, l, 2.0 ** -8)


@pytest.mark.parametrize("hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("window,n_first", WINDOWS)
def test_lengths(hq, hkv, dim, window, n_first):
    for i, lens in enumerate(LENS):
        run_and_check(Case8(lens, hq, hkv, dim, seed=100 + i), window, n_first)


@pytest.mark.parametrize("hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("pieces", ["2", "7"])
@pytest.mark.parametrize("tile", ["1", "2"])
def test_cut_tiles(hq, hkv, dim, pieces, tile, monkeypatch):
    monkeypatch.setenv("CALVO_ATTN_SPLITS", pieces)
    monkeypatch.setenv("CALVO_ROWS_TILE", tile)
    for window, n_first in [(5, 3), (64, 100), (300, 17), (FULL, 0)]:
        run_and_check(Case8([(100, 1), (0, 33), (257, 70)], hq, hkv, dim, seed=7), window, n_first)
    run_and_check(Case8([(400, 1), (700, 1)], hq, hkv, dim, seed=7), FULL, 0)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_long_context(dim):
    run_and_check(Case8([(6007, 1), (3001, 40), (20011, 2)], 8, 2, dim, seed=3), 2500, 100)
    run_and_check(Case8([(6007, 1)], 16, 2, dim, seed=4, layers=2), FULL, 0)
    run_and_check(Case8([(3000, 150)], 8, 2, dim, seed=5), FULL, 0)


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
            run_and_check(Case8(lens, hq, hkv, 128, seed=300 + i), window, n_first)


@pytest.mark.parametrize("variant", ["3", "4", "5"])
def test_long_contexts_of_128_wide_heads(variant, monkeypatch):
    """The steady loop with and without whole sub-tiles of first tokens in front."""
    monkeypatch.setenv("CALVO_ATTN_VARIANT", variant)
    for window, n_first in [(1000, 0), (1300, 300), (777, 1), (FULL, 0)]:
        run_and_check(Case8([(6007, 40), (2048, 2)], 8, 2, 128, seed=31), window, n_first)


def test_scale():
    c = Case8([(50, 20)], seed=5)
    wh.check_attn(c, c.run(30, 2, scale=0.5), 30, 2, scale=0.5, weight_step=2.0 ** -8)


def test_large_and_small_values():
    for size in (-60.0, 4.0):
        c = Case8([(208, 16), (96, 16)], 8, 2, 128, seed=21, size=size)
        c.k *= 2.0 ** size
        c.v *= 2.0 ** size
        run_and_check(c, FULL, 0)


@pytest.mark.parametrize("variant", ["3", "4", "5"])
def test_scores_that_grow_along_the_sequence(variant, monkeypatch):
    """The softmax reference moves in every step, by a little and by a lot."""
    monkeypatch.setenv("CALVO_ATTN_VARIANT", variant)
    for slope in (0.02, 0.3, -0.3):
        c = Case8([(500, 40)], 8, 2, 128, seed=31)
        k = np.ones((2, 16, 128)) * np.arange(1, 3)[:, None, None]
        n8 = 2 * 16 * 128
        for b, s in enumerate(c.tables[0][:32]):
            t = np.arange(16) + 16 * b
            x = k * (slope * t)[None, :, None]
            for h in range(2):
                sc = eo.least_scale(np.abs(x[h]).max())
                c.pool[0, s, h * 2048:(h + 1) * 2048] = eo.encode(x[h] / sc).reshape(-1)
                c.pool[0, s, 2 * n8 + 4 * h:2 * n8 + 4 * h + 4] = np.float32([sc]).view(np.uint8)
        run_and_check(c, FULL, 0)


# what a cached token may hold besides numbers: bytes of NaN, or a block whose scale is not finite
@pytest.mark.parametrize("hq,hkv,dim", [(8, 2, 128), (6, 2, 64), (4, 1, 256), (6, 3, 96)])
@pytest.mark.parametrize("what", ["k byte", "v byte", "both", "scale nan", "scale inf"])
@pytest.mark.parametrize("pieces", ["0", "3"])
@pytest.mark.parametrize("variant", ["3", "4", "5"])
def test_hidden_keys_do_not_reach_a_row(hq, hkv, dim, what, pieces, variant, monkeypatch):
    if variant != "5" and dim != 128:
        pytest.skip("one kernel only")
    monkeypatch.setenv("CALVO_ATTN_SPLITS", pieces)
    monkeypatch.setenv("CALVO_ATTN_VARIANT", variant)
    c = Case8([(150, 90)], hq, hkv, dim, seed=11)
    n8, t = c.hkv * 16 * dim, c.tables[0]
    window, n_first = 40, 5
    poisoned = [30, 120]
    for p in poisoned:
        s = t[p // 16]
        if what in ("k byte", "both"):
            c.pool[0, s, :n8].reshape(hkv, 16, dim)[:, p % 16, 3] = 0x7f
        if what in ("v byte", "both"):
            c.pool[0, s, n8:2 * n8].reshape(hkv, dim, 16)[:, 5, p % 16] = 0xff
        if what.startswith("scale"):
            c.pool[0, s, 2 * n8:2 * n8 + 8 * hkv] = np.full(2 * hkv, np.nan if what == "scale nan" else np.inf, np.float32).view(np.uint8)
    got = c.run(window, n_first)
    dead = np.unique(np.concatenate([np.arange(p // 16 * 16, p // 16 * 16 + 16) for p in poisoned])) if what.startswith("scale") else np.array(poisoned)
    sees = wh.wo.sees(range(150, 240), dead, window, n_first).any(axis=1)
    assert sees.any() and not sees.all()
    if what.startswith("scale"):                       # numbers for the oracle; no row that is compared sees them
        for b in {p // 16 for p in poisoned}:
            c.after[0, t[b], 2 * n8:2 * n8 + 8 * hkv] = np.ones(2 * hkv, np.float32).view(np.uint8)
    c.after[0][:, :2 * n8][(c.after[0][:, :2 * n8] & 127) == 127] = 0
    wh.check_attn(c, got, window, n_first, weight_step=2.0 ** -8, rows=~sees)
    out = got["out"][0].float()
    if what == "v byte":
        assert torch.isnan(out[torch.from_numpy(sees)][..., 5]).all() and torch.isfinite(out[..., :5]).all()
    else:
        assert torch.isnan(out[torch.from_numpy(sees)]).all()


def test_a_not_finite_query_stays_in_its_row():
    c = Case8([(90, 12)], 8, 2, 128, seed=13)
    c.q[0, 3, 2, 10] = float("nan")
    c.q[0, 7, 5, 1] = float("inf")
    got = c.run(FULL)
    rows = np.array([i not in (3, 7) for i in range(12)])
    wh.check_attn(c, got, FULL, 0, weight_step=2.0 ** -8, rows=rows)
    assert torch.isnan(got["out"][0, 3, 2].float()).all()
