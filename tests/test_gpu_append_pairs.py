"""Rotations whose pairs end inside a 16-byte chunk, into 8-bit pools; angles of every number of pairs, many tokens of a block at once."""
import numpy as np
import pytest

import e4m3_harness as eh
from e4m3_harness import Case8, inv_freq
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
