"""A long request among so many short ones that only its pieces leave partial results, on the GPU against the definition in 64 bits."""
import pytest

from e4m3_harness import Case8
from test_e4m3_plan import plan
from test_gpu_e4m3 import run_and_check
from window_harness import FULL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,dim", [(8, 8, 64), (32, 8, 64), (16, 8, 128), (8, 8, 256)])
@pytest.mark.parametrize("others", [140, 520])
def test_one_long_request(hq, hkv, dim, others):
    lens = [(5 * i % 61, 1) for i in range(others)]
    lens.insert(others // 2, (80 * others, 1))
    runs = plan(lens, hq, hkv, dim)[1]
    assert (runs[runs[:, 0] == others // 2, 6] > 1).all() and (runs[runs[:, 0] != others // 2, 6] == 1).all()
    run_and_check(Case8(lens, hq, hkv, dim, seed=17), FULL, 0)
