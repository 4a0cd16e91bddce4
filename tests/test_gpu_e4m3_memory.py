"""A context over an 8-bit pool takes no memory for calls that refuse it."""
import pytest
import torch

from paper_2603_21257_amd import binding as cb

pytestmark = pytest.mark.gpu


def taken(dim, dtype):
    """Device memory that a context takes besides the pool."""
    pool = torch.zeros(8 * cb.calvo_block_bytes(2, dim, dtype), dtype=torch.uint8, device="cuda:0")
    cb.calvo_destroy(cb.calvo_create(1, 4, 2, dim, dtype, 8, pool))          # what a device's first context leaves is there
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    ctx = cb.calvo_create(1, 4, 2, dim, dtype, 8, pool)
    after = torch.cuda.mem_get_info()[0]
    cb.calvo_destroy(ctx)
    return before - after


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_no_room_for_partial_results_of_causal_calls(dim):
    assert taken(dim, cb.CALVO_E4M3) < 8 << 20
    assert taken(dim, cb.CALVO_BF16) >= 32 << 20
