"""Rotations whose pairs end inside a 16-byte chunk, angles of every number of pairs, many tokens into 8-bit pools."""
import numpy as np
import pytest
import torch

import e4m3_harness as eh
from e4m3_harness import Case8, inv_freq
from paper_2603_21257_amd import binding as cb
from test_gpu_append import check_wide, run_wide
from window_harness import FULL, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,rot", [(48, 2), (48, 6), (64, 12), (64, 60), (80, 20), (96, 90), (128, 10), (128, 124), (256, 250), (160, 66)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_8_bit_pool(dim, rot, interleaved):
    for lens in ([(33, 6)], [(0, 16), (5, 40)], [(15, 1), (16, 1)]):
        print(f"[case] D={dim} rot={rot} {interleaved} {lens}", flush=True)
        c = Case8(lens, 4, 2, dim, seed=16)
        rope = (inv_freq(rot), rot, interleaved)
        got = c.run(FULL, rope=rope, far=np.arange(c.total) * 977 - 3)
        eh.check_append8(c, got, rope, np.arange(c.total) * 977 - 3)
        eh.check_q(c, got, rope, np.arange(c.total) * 977 - 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,rot", [(48, 6), (80, 20), (128, 10), (128, 124), (256, 250), (72, 66)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_wide_pools(dtype, dim, rot, interleaved):
    c = Case([(33, 6), (0, 17)], 4, 2, dim, dtype, seed=17)
    rope = (inv_freq(rot), rot, interleaved)
    check_wide(c, run_wide(c, rope), rope)


@pytest.mark.parametrize("dim,rot,interleaved", [(160, 160, False), (144, 40, True), (256, 20, False), (128, 128, False), (64, 12, False)])
def test_many_tokens_into_8_bits(dim, rot, interleaved):
    """More than sixteen tokens for every compute unit: rows of q of wide heads in a launch of their own, eight heads of a block to a workgroup, and several
    tokens of q to one where rows are narrow."""
    c = Case8([(7, 4500), (100, 1)], 4, 3, dim, seed=18)
    c.hq = 6
    c.q = c.q.repeat(1, 1, 2, 1)[:, :, :6].contiguous()
    rope = (inv_freq(rot), rot, interleaved)
    far = np.arange(c.total) * 31 + 5
    dev = "cuda:0"
    pool, q, k, v = torch.from_numpy(c.pool).to(dev), c.q.to(dev), c.k.to(dev), c.v.to(dev)
    q_out = torch.empty_like(q)
    r = cb.make_rope(torch.from_numpy(rope[0]).to(dev), rot, interleaved, torch.from_numpy(far.astype(np.int32)).to(dev))
    torch.cuda.synchronize()
    ctx = c.create(pool)
    plan = cb.calvo_window_prepare(ctx, c.requests(), FULL)
    cb.calvo_kv_append(plan, 0, k[0], v[0], q[0], q_out[0], r)
    cb.calvo_window_destroy(plan)
    cb.calvo_destroy(ctx)
    got = {"pool": pool.cpu().numpy(), "q": q_out.cpu()}
    eh.check_append8(c, got, rope, far)
    eh.check_q(c, got, rope, far)
