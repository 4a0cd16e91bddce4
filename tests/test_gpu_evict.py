"""Eviction by gathered weight on the GPU: the chosen positions, the moved bytes and what is left alone."""
import numpy as np
import pytest
import torch

from oracle import window_oracle as wo
from paper_2603_21257_amd import binding as cb

pytestmark = pytest.mark.gpu
B = 16


def run(lens, keeps, hkv=2, dim=64, dtype="bf16", layers=3, seed=1, special=True, with_out=True, layer_range=None):
    """lens: tokens; keeps: (n_keep, n_first, n_last)."""
    rng = np.random.default_rng(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    as_int = torch.int16 if dtype == "bf16" else torch.int32
    src_n, dst_n = [-(-n // B) for n in lens], [-(-k[0] // B) for k in keeps]
    slots = sum(src_n) + sum(dst_n) + 4
    perm = rng.permutation(slots).astype(np.int32)
    at, tables = 0, []
    for a, b in zip(src_n, dst_n):
        tables.append((perm[at:at + a], perm[at + a:at + a + b]))
        at += a + b
    pool = torch.randn((layers, slots, 2, B, hkv, dim), generator=torch.Generator().manual_seed(seed)).to(dt)
    l0, l1 = layer_range or (0, layers)
    R, stride, kstride, ostride = len(lens) + 2, max(lens) + 5, max(k[0] for k in keeps) + 3, max(k[0] for k in keeps) + 1
    mass = rng.exponential(size=(l1 - l0, R, hkv, stride)).astype(np.float32)
    if special:
        u = rng.random(mass.shape)
        mass[u < 0.3] = 0.0
        mass[(u > 0.3) & (u < 0.35)] = -0.0
        mass[(u > 0.35) & (u < 0.5)] = 0.5
        mass[(u > 0.5) & (u < 0.52)] = np.nan
        mass[(u > 0.52) & (u < 0.54)] = np.inf
        mass[(u > 0.54) & (u < 0.56)] = -np.inf
        mass[(u > 0.56) & (u < 0.6)] = 1e-42
        mass[(u > 0.6) & (u < 0.65)] = -1.5
    rows = rng.permutation(R)[:len(lens)]
    d_pool, d_mass = pool.to("cuda:0"), torch.from_numpy(mass).to("cuda:0")
    kept = torch.full((l1 - l0, len(lens), hkv, kstride), -7, dtype=torch.int32, device="cuda:0")
    out = torch.full((l1 - l0, R, hkv, ostride), -7.0, device="cuda:0")
    torch.cuda.synchronize()
    ctx = cb.calvo_create(layers, hkv, hkv, dim, cb.CALVO_BF16 if dtype == "bf16" else cb.CALVO_F32, slots, d_pool)
    try:
        reqs = [cb.make_evict_request(s, n, d, k[0], k[1], k[2], int(r)) for n, k, (s, d), r in zip(lens, keeps, tables, rows)]
        cb.calvo_kv_evict(ctx, reqs, l0, l1, d_mass, R, stride, kept, kstride, out if with_out else None, ostride if with_out else 0)
    finally:
        cb.calvo_destroy(ctx)
    torch.cuda.synchronize()
    want_pool, want_kept, want_out = pool.clone(), torch.full_like(kept.cpu(), -7), torch.full_like(out.cpu(), -7.0)
    for l in range(l0, l1):
        for r, (n, k, (s, d)) in enumerate(zip(lens, keeps, tables)):
            for g in range(hkv):
                at = wo.choose(mass[l - l0, rows[r], g], n, *k)
                want_kept[l - l0, r, g, :k[0]] = torch.from_numpy(at)
                if with_out:
                    want_out[l - l0, rows[r], g, :k[0]] = torch.from_numpy(mass[l - l0, rows[r], g][at])
                j = np.arange(k[0])
                for half in (0, 1):
                    want_pool[l, d[j // B], half, j % B, g] = pool[l, s[at // B], half, at % B, g]
    assert torch.equal(kept.cpu(), want_kept)
    assert torch.equal(out.cpu().view(torch.int32), want_out.view(torch.int32))
    assert torch.equal(d_pool.cpu().view(as_int), want_pool.view(as_int))


@pytest.mark.parametrize("n,keep", [(1, (1, 0, 0)), (1, (1, 1, 0)), (17, (16, 0, 0)), (17, (17, 3, 4)), (64, (10, 2, 8)), (100, (33, 4, 16)), (1000, (1, 0, 0)),
                                    (1025, (512, 0, 100)), (3001, (900, 10, 0)), (5000, (4999, 0, 0)), (2048, (300, 300, 0)), (2048, (300, 100, 200))])
@pytest.mark.parametrize("special", [True, False])
def test_lengths(n, keep, special):
    run([n], [keep], special=special, seed=n)


@pytest.mark.parametrize("hkv,dim,dtype", [(1, 8, "bf16"), (3, 40, "bf16"), (8, 128, "bf16"), (2, 256, "bf16"), (2, 8, "f32"), (3, 96, "f32"), (2, 256, "f32")])
def test_shapes_and_batches(hkv, dim, dtype):
    run([70, 300, 16, 1500], [(20, 2, 3), (300, 0, 0), (0, 0, 0), (77, 4, 30)], hkv, dim, dtype, seed=dim)
    run([333], [(48, 4, 16)], hkv, dim, dtype, layers=4, layer_range=(1, 3), with_out=False, seed=3)


def test_long():
    run([40000, 20011], [(5000, 4, 256), (20011, 0, 0)], hkv=4, dim=64, layers=2, seed=2)
