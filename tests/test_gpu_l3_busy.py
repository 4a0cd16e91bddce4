"""What calvo_l3_wait says of the emulated link while the loader's thread is held up between two chunks."""
import pytest
import torch

import hip_harness as hh
from paper_2603_21257_amd import binding as cb
from paper_2603_21257_amd import workload as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("delay_us", ["0", "2000"])
def test_the_link_is_occupied_while_a_chunk_is_handed_over(delay_us, monkeypatch):
    """16 chunks of 4.2 ms at 1 GB/s, each handed over with a delay on the host that is shorter than a chunk: the link streams on its own, and is occupied for as
    long as the bytes take."""
    monkeypatch.setenv("CALVO_INGEST_DELAY_US", delay_us)
    shape = wl.Shape(2, 8, 8, 128, "bf16", 600)              # 64 KiB blocks
    w = wl.make_custom(shape, [(512 * 16, 16)], seed=5)
    s = w.shape
    pool = hh.to_torch(hh.sentinel_pool_np(s), s, torch.device("cuda:0"))
    remote = hh.to_torch(w.host_kv, s)
    ctx = cb.calvo_create(s.n_layers, s.n_q_heads, s.n_kv_heads, s.head_dim, cb.CALVO_BF16, s.pool_blocks, pool, staging_bytes=8 << 20)
    try:
        cb.calvo_kv_ingest_l3(ctx, hh.make_requests(w, remote), 0, 2, chunk_bytes=4 << 20, n_slots=8, n_threads=2, l3_GBps=1.0)
        st = cb.calvo_l3_wait(ctx)
    finally:
        cb.calvo_destroy(ctx)
    print(f"busy {st['l3_busy_s'] * 1e3:.2f} ms of {st['total_s'] * 1e3:.2f}, ring wait {st['ring_wait_s'] * 1e3:.2f} ms", flush=True)
    assert st["l3_busy_s"] >= w.ingest_bytes() / 1e9 * 0.98
    assert st["l3_busy_s"] <= st["total_s"] + 1e-4
