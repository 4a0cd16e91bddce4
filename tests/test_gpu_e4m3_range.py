"""8-bit pools at the ends of bf16's range: new values near the largest, and below the least normal one."""
import numpy as np
import pytest
import torch

import e4m3_harness as eh
from e4m3_harness import Case8
from oracle import e4m3_oracle as eo
from window_harness import FULL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 128), (2, 1, 48), (8, 2, 256)])
def test_values_near_the_largest(hq, hkv, dim):
    """The scale is 2^120 where a value is above 448 * 2^119.  A single token sees itself alone: its output is V as it is held, which bf16 has exactly."""
    c = Case8([(0, 1), (0, 1)], hq, hkv, dim, seed=4)
    gen = np.random.default_rng(4)
    c.v = torch.from_numpy(gen.choice([1.8125, -1.8125, 1.875, 1.0, -0.5, 0.0], (1, 2, hkv, dim)) * 2.0 ** 127).to(torch.bfloat16)
    c.v[..., 0] = 1.875 * 2.0 ** 127
    got = c.run(FULL)
    eh.check_append8(c, got)
    for r, t in enumerate(c.tables):
        assert (eo.parts(got["pool"][0], hkv, dim)[2][t[0], 1] == 2.0 ** 120).all()
        held = eo.widened(got["pool"][0], hkv, dim)[t[0], 1, 0]
        assert np.array_equal(got["out"][0, r].double().numpy(), np.repeat(held, hq // hkv, axis=0))


def test_values_below_the_least_normal_one():
    """The scale stays at 2^-126; bytes by the definition, and outputs within 2^-126 of what they stand for."""
    c = Case8([(0, 1), (0, 3)], 4, 2, 64, seed=6)
    c.k = (c.k.double() * 2.0 ** -127).to(torch.bfloat16)
    c.v = (c.v.double() * 2.0 ** -127).to(torch.bfloat16)
    got = c.run(FULL)
    eh.check_append8(c, got)
    assert (eo.parts(got["pool"][0], 2, 64)[2][[t[0] for t in c.tables]] == 2.0 ** -126).all()
    held = eo.widened(got["pool"][0], 2, 64)[c.tables[0][0], 1, 0]
    assert (np.abs(got["out"][0, 0].double().numpy() - np.repeat(held, 2, axis=0)) <= 2.0 ** -126).all()
    # three tokens whose scores are below 2^-120: their weights are equal
    held = eo.widened(got["pool"][0], 2, 64)[c.tables[1][0], 1, :3]
    for i in range(3):
        want = np.repeat(held[:i + 1].mean(axis=0), 2, axis=0)
        assert (np.abs(got["out"][0, 1 + i].double().numpy() - want) <= 2.0 ** -126 + 2.0 ** -7 * np.abs(want)).all()
