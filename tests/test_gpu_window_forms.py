"""Forms of the window operators' calls beside those of test_gpu_window.py, test_gpu_mass.py and test_gpu_evict.py: requests that share cached blocks, the smallest heads,
more head layouts, large scores, weights that are all alike."""
import numpy as np
import pytest
import torch

import test_gpu_evict
import window_harness as wh
from oracle import window_oracle as wo
from paper_2603_21257_amd import binding as cb
from window_harness import FULL, Case

pytestmark = pytest.mark.gpu


class Shared(Case):
    """Every request's first `blocks` blocks are the first one's."""

    def __init__(self, blocks, lens, *a, **k):
        super().__init__(lens, *a, **k)
        assert all(c >= 16 * blocks for c, _ in lens)
        for t in self.tables[1:]:
            t[:blocks] = self.tables[0][:blocks]


def check(c, window, n_first, mass_too=True, last_rows=0, scale=0.0, scores=None):
    print(f"[case] {c.dtype} {c.hq}/{c.hkv} D={c.dim} {c.lens} window={window} first={n_first} last={last_rows}", flush=True)
    m = torch.rand((c.layers, len(c.lens) + 1, c.hkv, c.stride()), generator=torch.Generator().manual_seed(5)) if mass_too else None
    got = c.run(window, n_first, mass=mass_too, last_rows=last_rows, mass_in=m, scale=scale)
    wh.check_pool(c, got)
    for l in range(c.layers):
        wh.check_attn(c, got, window, n_first, l, 2.0 ** -8 if (c.dtype, c.dim) == ("bf16", 128) else 0.0, scale=scores)
        if mass_too:
            wh.check_mass(c, got, window, n_first, last_rows, m, l, scale=scores)


@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 128), ("bf16", 32, 8, 128), ("bf16", 8, 2, 64), ("bf16", 4, 2, 40), ("f32", 8, 2, 64), ("f32", 4, 1, 256)])
@pytest.mark.parametrize("lens", [[(49, 1), (70, 1), (48, 1), (300, 1)], [(64, 20), (48, 3), (90, 0), (51, 1)], [(500, 130), (48, 1), (200, 1)]])
def test_requests_that_share_cached_blocks(dtype, hq, hkv, dim, lens):
    for window, n_first in [(30, 4), (300, 0), (FULL, 0)]:
        check(Shared(3, lens, hq, hkv, dim, dtype, seed=81, layers=2), window, n_first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 8), (1, 1, 8), (6, 2, 16), (8, 1, 24), (4, 4, 32), (3, 1, 56), (4, 2, 72), (2, 1, 136), (2, 2, 248)])
def test_small_and_odd_heads(dtype, hq, hkv, dim):
    for lens in [[(0, 1)], [(33, 1), (700, 1)], [(17, 3), (0, 0), (40, 0), (0, 2)], [(100, 1), (0, 33), (257, 70)]]:
        for window, n_first in [(5, 3), (64, 20), (FULL, 0)]:
            check(Case(lens, hq, hkv, dim, dtype, seed=82), window, n_first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,dim", [(1, 1, 128), (3, 3, 128), (7, 1, 128), (16, 16, 128), (64, 1, 128), (48, 2, 64), (32, 16, 64), (100, 1, 64), (14, 2, 128), (128, 1, 8)])
def test_head_layouts(dtype, hq, hkv, dim):
    for lens in [[(40, 1), (500, 1)], [(17, 3), (250, 40)]]:
        for window, n_first in [(33, 5), (FULL, 0)]:
            for last_rows in (0, 2):
                check(Case(lens, hq, hkv, dim, dtype, seed=83), window, n_first, last_rows=last_rows)


@pytest.mark.parametrize("dtype,hq,hkv,dim", [("bf16", 8, 2, 128), ("bf16", 8, 2, 64), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("scale", [2.0 ** -20, 1.5, 30.0])
def test_flat_and_steep_scores(dtype, hq, hkv, dim, scale):
    """From weights that are all alike to rows that one key has to itself.  (Gathered weights: their bound takes an error of an exponent for one of the
    weight, which the steepest scores are too large for.)"""
    for lens in [[(500, 1), (33, 1)], [(300, 90)]]:
        check(Case(lens, hq, hkv, dim, dtype, seed=84), 200, 4, mass_too=scale < 30, scale=scale, scores=float(np.float32(scale)))


@pytest.mark.parametrize("value", [0.0, 1.0, -2.5, float("nan"), float("inf"), -float("inf"), 1e-45])
@pytest.mark.parametrize("n,keep,first,last", [(300, 17, 0, 0), (5000, 1234, 3, 100), (40000, 39000, 1, 1)])
def test_eviction_of_weights_that_are_all_alike(value, n, keep, first, last):
    """Ties all the way: the first of the tokens that are chosen from stay."""
    dst, src, hkv = -(-keep // 16), -(-n // 16), 2
    pool = torch.randn((1, src + dst, 2, 16, hkv, 8), generator=torch.Generator().manual_seed(1)).to("cuda:0")
    was = pool.clone()
    mass = torch.full((1, 1, hkv, n), value, device="cuda:0")
    kept = torch.full((1, 1, hkv, keep), -7, dtype=torch.int32, device="cuda:0")
    torch.cuda.synchronize()
    ctx = cb.calvo_create(1, hkv, hkv, 8, cb.CALVO_F32, src + dst, pool)
    try:
        cb.calvo_kv_evict(ctx, [cb.make_evict_request(np.arange(src), n, np.arange(src, src + dst), keep, first, last)], 0, 1, mass, 1, n, kept, keep)
    finally:
        cb.calvo_destroy(ctx)
    torch.cuda.synchronize()
    want = np.concatenate([np.arange(keep - last), np.arange(n - last, n)])
    if n == 300:
        assert np.array_equal(want, wo.choose(mass[0, 0, 0].cpu().numpy(), n, keep, first, last))
    for g in range(hkv):
        assert np.array_equal(kept[0, 0, g].cpu().numpy(), want)
    j, at = torch.arange(keep), torch.from_numpy(want)
    assert torch.equal(pool[0, src + j // 16, :, j % 16], was[0, at // 16, :, at % 16])
    assert torch.equal(pool[0, :src], was[0, :src])


def test_eviction_of_short_requests_beside_a_long_one():
    """The long request sets how many positions a wave holds; the others have a part of them."""
    test_gpu_evict.run([40000, 1, 17, 300, 1025, 5000], [(100, 1, 2), (1, 0, 0), (9, 0, 3), (299, 4, 16), (1, 0, 0), (4096, 0, 0)], hkv=3, dim=8, layers=2, seed=85)


def test_captured_calls_and_loads(monkeypatch):
    """While a layer is loaded a captured call for it is refused and the capture goes on; once it is in, the same call is taken, and the graph does what the
    eager call does."""
    monkeypatch.setenv("CALVO_TEST_SCATTER_DELAY_US", "20000")
    L = 6
    c = Case([(320, 1)], 8, 2, 128, seed=86, layers=L)
    host = torch.empty((L, 20, 2, 16, 2, 128), dtype=c.dt, pin_memory=True)
    host.copy_(c.pool[:, c.tables[0][:20].tolist()])
    stream = torch.cuda.Stream()
    pool = torch.full(c.pool.shape, float("nan"), dtype=c.dt, device="cuda:0")
    q, k, v = (x.to("cuda:0") for x in (c.q, c.k, c.v))
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:-1], device="cuda:0")
    mass = torch.zeros((L, 1, 2, 321), device="cuda:0")
    torch.cuda.synchronize()
    ctx = cb.calvo_create(L, 8, 2, 128, cb.CALVO_BF16, c.slots, pool, staging_bytes=1 << 20, compute_stream=stream.cuda_stream)

    def calls(l):
        cb.calvo_window_attn(plan, l, q[l], k[l], v[l], out[l], lse[l])
        cb.calvo_attn_mass(plan, l, q[l], lse[l], None, mass[l], 1, 321)

    try:
        plan = cb.calvo_window_prepare(ctx, c.requests(), 200, 4)
        torch.cuda.synchronize()
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        one = torch.zeros(1, device="cuda:0")
        torch.cuda.synchronize()
        for when, graph in zip(("under way", "in"), graphs):
            with torch.cuda.stream(stream):
                if when == "under way":
                    cb.calvo_kv_ingest(ctx, [cb.make_request(host, host[0].numel() * 2, c.tables[0], 20, 0)], 0, L)
                graph.capture_begin()
                if when == "under way":
                    with pytest.raises(cb.CalvoError) as e:
                        calls(L - 1)
                    assert e.value.code == cb.CALVO_ENOTREADY, e.value
                    one.add_(1)
                else:
                    for l in range(L):
                        calls(l)
                graph.capture_end()
            torch.cuda.synchronize()
        for graph in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
            torch.cuda.synchronize()
        assert one.item() == 1
        got = [x.clone() for x in (out, lse, mass)]
        for x in (out, lse, mass):
            x.zero_()
        torch.cuda.synchronize()
        for l in range(L):
            calls(l)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, mass)))
        del graphs, graph
        cb.calvo_window_destroy(plan)
    finally:
        cb.calvo_destroy(ctx)
    for l in range(L):
        wh.check_attn(c, {"out": out.cpu(), "lse": lse.cpu()}, 200, 4, l, 2.0 ** -8)
