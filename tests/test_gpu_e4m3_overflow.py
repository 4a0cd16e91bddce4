"""Values of an 8-bit pool that bf16 reads as infinite - 256 times a scale of 2^120 and more - reach the rows that see them and no others."""
import numpy as np
import pytest
import torch

import e4m3_harness as eh
import window_harness as wh
from e4m3_harness import Case8
from oracle import e4m3_oracle as eo
from window_harness import FULL

pytestmark = pytest.mark.gpu

ROWS = [("5", "0", "1"), ("5", "0", "2"), ("5", "3", "1")]   # CALVO_ATTN_VARIANT: 5 the packed rows, 3 and 4 the pipelined kernels, of 128-wide heads alone
PIPELINED = [("3", "0", "0"), ("4", "0", "0"), ("4", "3", "0")]
CASES = [(*shape, *how) for shape in ((8, 2, 128), (6, 2, 64), (4, 1, 256), (6, 3, 96), (8, 8, 48)) for how in ROWS + PIPELINED * (shape[2] == 128)]


def forced(monkeypatch, variant, pieces, tile):
    monkeypatch.setenv("CALVO_ATTN_VARIANT", variant)
    monkeypatch.setenv("CALVO_ATTN_SPLITS", pieces)
    monkeypatch.setenv("CALVO_ROWS_TILE", tile)


@pytest.mark.parametrize("hq,hkv,dim,variant,pieces,tile", CASES)
@pytest.mark.parametrize("byte", [0x7e, 0xf8])
def test_cached_values(hq, hkv, dim, byte, variant, pieces, tile, monkeypatch):
    """A block of V at scale 2^120 whose only byte that is not zero stands for +-448 or -256 times it, at one token and element."""
    forced(monkeypatch, variant, pieces, tile)
    c = Case8([(150, 90)], hq, hkv, dim, seed=11)
    n8, t, window, n_first, poisoned = hkv * 16 * dim, c.tables[0], 40, 5, np.array([30, 120])
    for p in poisoned:
        s = t[p // 16]
        v = np.zeros((hkv, dim, 16), np.uint8)
        v[:, 5, p % 16] = byte
        c.pool[0, s, n8:2 * n8] = v.reshape(-1)
        c.pool[0, s, 2 * n8 + 4 * hkv:2 * n8 + 8 * hkv] = np.full(hkv, 2.0 ** 120, np.float32).view(np.uint8)
    got = c.run(window, n_first)
    sees = wh.wo.sees(range(150, 240), poisoned, window, n_first).any(axis=1)
    assert sees.any() and not sees.all()
    wh.check_attn(c, got, window, n_first, weight_step=2.0 ** -8, rows=~sees)
    out = got["out"][0].float()[torch.from_numpy(sees)]
    assert not torch.isfinite(out[..., 5]).any() and torch.isfinite(out[..., :5]).all() and torch.isfinite(out[..., 6:]).all()


@pytest.mark.parametrize("hq,hkv,dim,variant,pieces,tile", CASES)
@pytest.mark.parametrize("value", [torch.finfo(torch.bfloat16).max, 1.9375 * 2.0 ** 127, -1.9375 * 2.0 ** 127])
def test_appended_values(hq, hkv, dim, value, variant, pieces, tile, monkeypatch):
    """A chunk whose last token's V is finite in bf16 and rounds to 256 times the scale of 2^120: the last row alone is not finite there."""
    forced(monkeypatch, variant, pieces, tile)
    c = Case8([(20, 30)], hq, hkv, dim, seed=12)
    c.v[0, -1, :, 7] = value
    got = c.run(FULL)
    eh.check_append8(c, got)
    scale, held = eo.parts(got["pool"][0], hkv, dim)[2], eo.widened(got["pool"][0], hkv, dim)
    assert (scale[c.tables[0][-1], 1] == 2.0 ** 120).all() and (np.abs(held[c.tables[0][-1], 1, 49 % 16, :, 7]) == 2.0 ** 128).all()
    wh.check_attn(c, got, FULL, weight_step=2.0 ** -8, rows=np.arange(30) < 29)
    assert not torch.isfinite(got["out"][0, 29, :, 7].float()).any()


def test_single_tokens_behind_a_window(monkeypatch):
    """Tokens that have left the window, in the blocks and steps that its first ones are in."""
    for dim, pieces in ((128, "0"), (128, "4"), (64, "0"), (256, "2")):
        monkeypatch.setenv("CALVO_ATTN_SPLITS", pieces)
        c = Case8([(200, 1), (511, 1), (70, 1)], 8, 2, dim, seed=13)
        n8 = 2 * 16 * dim
        for (n, _), t in zip(c.lens, c.tables):
            p = n - 48                                       # the window of 48 begins behind it
            v = np.zeros((2, dim, 16), np.uint8)
            v[:, :, p % 16] = 0x7e
            c.pool[0, t[p // 16], n8:2 * n8] = v.reshape(-1)
            c.pool[0, t[p // 16], 2 * n8 + 8:2 * n8 + 16] = np.full(2, 2.0 ** 120, np.float32).view(np.uint8)
        got = c.run(48)
        wh.check_attn(c, got, 48, weight_step=2.0 ** -8)
