"""The append with rotation (calvo_kv_append) on the GPU against the definition in 64 bits, pools of every type."""
import numpy as np
import pytest
import torch

import e4m3_harness as eh
from e4m3_harness import Case8, inv_freq
from oracle import e4m3_oracle as eo
from paper_2603_21257_amd import binding as cb
from window_harness import FULL, OUT, Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

LENS = [[(0, 1)], [(15, 1)], [(16, 1)], [(31, 3), (0, 0), (40, 0), (0, 2)], [(100, 1), (0, 33), (257, 70), (5, 11)], [(0, 16)], [(47, 1)]]
ROPES = [(1.0, False), (1.0, True), (0.5, False), (0.25, True), (0.0, False)]    # share of a head that is rotated
SHAPES = [(8, 2, 64), (8, 2, 128), (5, 1, 128), (6, 3, 96), (8, 8, 48), (4, 1, 256), (6, 2, 208), (32, 8, 128), (2, 2, 16)]


def rope_of(dim, share, interleaved):
    rot = int(dim * share) // 2 * 2
    return (inv_freq(rot), rot, interleaved) if rot else None


@pytest.mark.parametrize("hq,hkv,dim", SHAPES)
@pytest.mark.parametrize("share,interleaved", ROPES)
def test_8_bit_pool(hq, hkv, dim, share, interleaved):
    rope = rope_of(dim, share, interleaved)
    for i, lens in enumerate(LENS):
        print(f"[case] {hq}/{hkv} D={dim} {lens} {share} {interleaved}", flush=True)
        c = Case8(lens, hq, hkv, dim, seed=50 + i, layers=2)
        far = np.random.default_rng(i).integers(-5, 3000000, c.total) if i % 2 else None
        got = c.run(FULL, rope=rope, far=far)
        eh.check_append8(c, got, rope, far if rope else None)
        if rope:
            eh.check_q(c, got, rope, far)


def test_scales_grow_and_stay():
    """New values far above, far below and within what the block holds; a block whose tokens are all zero."""
    for size in (-20.0, 20.0, 0.0, -100.0, 90.0):
        c = Case8([(3, 1), (9, 5), (15, 20), (0, 4)], 4, 2, 64, seed=9, size=size)
        eh.check_append8(c, c.run(FULL))
    c = Case8([(3, 2), (0, 3)], 4, 2, 64, seed=9)
    c.k.zero_()
    c.v[:, :, 1] = 0
    eh.check_append8(c, c.run(FULL))


def test_token_by_token():
    """Sixteen steps into one block: every step by the definition on what the one before left."""
    gen = torch.Generator().manual_seed(5)
    c = Case8([(0, 1)], 4, 2, 128, seed=2)
    for i in range(18):
        c.lens = [(i, 1)]
        if i == 16:
            c.tables = [np.concatenate([c.tables[0], np.setdiff1d(np.arange(c.slots, dtype=np.int32), c.tables[0])[:1]])]
        c.k = (torch.randn((1, 1, 2, 128), generator=gen) * 2.0 ** (i % 5 - 2)).to(c.dt)
        c.v = (torch.randn((1, 1, 2, 128), generator=gen) * 2.0 ** (i % 7 - 3)).to(c.dt)
        got = c.run(FULL)
        eh.check_append8(c, got)
        c.pool = got["pool"].copy()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite(value):
    c = Case8([(20, 3), (0, 5)], 4, 2, 64, seed=3)
    c.k[0, 1, 0, 7] = value
    c.v[0, 4, 1, 63] = value
    got = c.run(FULL)
    eh.check_append8(c, got)
    scale = eo.parts(got["pool"][0], 2, 64)[2]
    assert np.isnan(scale[c.tables[0][1], 0, 0]) and np.isfinite(scale[c.tables[0][1], 0, 1]) and np.isnan(scale[c.tables[1][0], 1, 1])


def run_wide(c, rope, far=None, fused=False, with_q=True, with_kv=True):
    """calvo_kv_append on a bf16 or fp32 pool, one layer at a time."""
    pool = c.pool.to(DEV)
    if fused:
        rows = torch.cat([x.reshape(c.layers, c.total, -1) for x in (c.q, c.k, c.v)], dim=-1).to(DEV)
        q, k, v = (x.unflatten(-1, (-1, c.dim)) for x in rows.split([c.hq * c.dim, c.hkv * c.dim, c.hkv * c.dim], dim=-1))
    else:
        q, k, v = (x.to(DEV) for x in (c.q, c.k, c.v))
    q_out = torch.full((c.layers, c.total + 4, c.hq, c.dim), 7.0, dtype=c.dt, device=DEV)
    r = None
    if rope:
        r = cb.make_rope(torch.from_numpy(rope[0]).to(DEV), rope[1], rope[2], None if far is None else torch.from_numpy(far.astype(np.int32)).to(DEV))
    torch.cuda.synchronize()
    ctx = c.create(pool)
    try:
        plan = cb.calvo_window_prepare(ctx, c.requests(), FULL)
        for l in range(c.layers):
            cb.calvo_kv_append(plan, l, k[l] if with_kv else None, v[l] if with_kv else None, q[l] if with_q else None, q_out[l] if with_q else None, r,
                               k.stride(1), v.stride(1), q.stride(1))
        cb.calvo_window_destroy(plan)
    finally:
        cb.calvo_destroy(ctx)
    torch.cuda.synchronize()
    assert (q_out[:, c.total:].float() == 7.0).all()
    return {"q": q_out[:, :c.total].cpu(), "pool": pool.cpu()}


def check_wide(c, got, rope, far=None, with_q=True, with_kv=True):
    pos = np.concatenate([np.arange(a, a + n) for a, n in c.lens]) if far is None else far
    as_int = torch.int16 if c.dtype == "bf16" else torch.int32
    want = c.pool.clone()
    for l in range(c.layers):
        for src, name in ((c.q, "q"), (c.k, "k")):
            x = src[l].double().numpy()
            y = eo.rotate(x, pos, *rope) if rope else x
            tol = (eh.rotation_error(x, pos, rope[1]) * (1 + OUT[c.dtype]) if rope else 0) + (OUT[c.dtype] * np.abs(y) + 1e-38 if rope else 0)
            if name == "q":
                if with_q:
                    assert (np.abs(got["q"][l].double().numpy() - y) <= tol).all()
                continue
            for r, ((a, n), t) in enumerate(zip(c.lens, c.tables)):
                for i in range(n if with_kv else 0):
                    slot, p, row = t[(a + i) // 16], (a + i) % 16, c.cu[r] + i
                    held = got["pool"][l, slot, 0, p].double().numpy()
                    assert (np.abs(held - y[row]) <= np.broadcast_to(tol, y.shape)[row]).all()
                    if rope:                                     # elements that are not rotated keep their bits
                        assert torch.equal(got["pool"][l, slot, 0, p, :, rope[1]:], c.k[l, row, :, rope[1]:])
                    want[l, slot, 0, p], want[l, slot, 1, p] = got["pool"][l, slot, 0, p], c.v[l, row]
    assert torch.equal(got["pool"].view(as_int), want.view(as_int))


@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 128), ("bf16", 6, 3, 96), ("bf16", 8, 8, 40), ("bf16", 4, 1, 256), ("bf16", 2, 1, 8),
                                              ("f32", 8, 2, 64), ("f32", 6, 3, 40), ("f32", 5, 1, 128), ("f32", 4, 2, 256)])
@pytest.mark.parametrize("share,interleaved", ROPES)
def test_wide_pools(dtype, hq, hkv, dim, share, interleaved):
    rope = rope_of(dim, share, interleaved)
    for i, lens in enumerate(LENS):
        print(f"[case] {dtype} {hq}/{hkv} D={dim} {lens} {share} {interleaved}", flush=True)
        c = Case(lens, hq, hkv, dim, dtype, seed=70 + i, layers=2)
        far = np.random.default_rng(i).integers(-5, 3000000, c.total) if i % 2 else None
        check_wide(c, run_wide(c, rope, far, fused=i % 3 == 0), rope, far)


def test_many_tokens():
    """More than sixteen tokens for every compute unit: a workgroup takes several."""
    for dtype, dim in (("bf16", 64), ("f32", 32)):
        rope = rope_of(dim, 1.0, False)
        c = Case([(7, 4500), (100, 1)], 4, 1, dim, dtype, seed=8)
        check_wide(c, run_wide(c, rope), rope)
    c = Case8([(7, 4500), (100, 1)], 4, 2, 64, seed=8)
    rope = rope_of(64, 1.0, False)
    pool, q = torch.from_numpy(c.pool).to(DEV), c.q.to(DEV)
    k, v, q_out = c.k.to(DEV), c.v.to(DEV), torch.empty_like(q)
    torch.cuda.synchronize()
    ctx = c.create(pool)
    plan = cb.calvo_window_prepare(ctx, c.requests(), FULL)
    cb.calvo_kv_append(plan, 0, k[0], v[0], q[0], q_out[0], cb.make_rope(torch.from_numpy(rope[0]).to(DEV), 64))
    cb.calvo_window_destroy(plan)
    cb.calvo_destroy(ctx)
    got = {"pool": pool.cpu().numpy(), "q": q_out.cpu()}
    eh.check_append8(c, got, rope)
    eh.check_q(c, got, rope)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_the_call(dtype):
    """q alone, K and V alone; far positions, the last that fit 32 bits and negative ones."""
    c = Case([(17, 5), (64, 2)], 8, 2, 64, dtype, seed=4)
    rope = rope_of(64, 1.0, False)
    check_wide(c, run_wide(c, rope, with_kv=False), rope, with_kv=False)
    check_wide(c, run_wide(c, rope, with_q=False), rope, with_q=False)
    far = np.array([2 ** 31 - 1, -2 ** 31, 0, 1, -1, 2 ** 30 + 7, 123456789])
    check_wide(c, run_wide(c, rope, far), rope, far)


def test_rotation_of_pairs_whose_halves_are_not_whole_chunks():
    for dim, rot in ((40, 20), (64, 12), (96, 90), (24, 2)):
        for dtype in ("bf16", "f32"):
            for inter in (False, True):
                c = Case([(33, 6)], 4, 2, dim, dtype, seed=6)
                rope = (inv_freq(rot), rot, inter)
                check_wide(c, run_wide(c, rope), rope)
    for dim, rot in ((48, 20), (64, 12), (96, 90), (16, 2)):
        c = Case8([(33, 6)], 4, 2, dim, seed=6)
        rope = (inv_freq(rot), rot, False)
        got = c.run(FULL, rope=rope)
        eh.check_append8(c, got, rope)
        eh.check_q(c, got, rope)
