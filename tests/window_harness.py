"""Test-side driver of the window operators: a pool whose unused rows are NaN, random tables, and both sides of a comparison."""
import numpy as np
import torch

from oracle import window_oracle as wo
from paper_2603_21257_amd import binding as cb

B = 16
FULL = (1 << 31) - 1
U32 = 2.0 ** -24                       # half a step of fp32, relative
OUT = {"bf16": 2.0 ** -8, "f32": U32}  # of the stored type


class Case:
    """One layer of a pool, requests of (n_cached, n_new) tokens, q and the new K and V."""

    def __init__(self, lens, hq=8, hkv=2, dim=64, dtype="bf16", seed=1, spare=5, layers=1):
        rng = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.dim, self.dtype, self.layers = lens, hq, hkv, dim, dtype, layers
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        blocks = [-(-(c + n) // B) for c, n in lens]
        self.slots = sum(blocks) + spare
        perm = rng.permutation(self.slots).astype(np.int32)
        at = np.cumsum([0] + blocks)
        self.tables = [perm[a:b].copy() for a, b in zip(at[:-1], at[1:])]
        self.free = perm[at[-1]:]
        gen = torch.Generator().manual_seed(seed)
        self.pool = torch.full((layers, self.slots, 2, B, hkv, dim), float("nan"), dtype=self.dt)
        for (c, n), t in zip(lens, self.tables):
            for p in range(c):
                self.pool[:, t[p // B], :, p % B] = torch.randn((layers, 2, hkv, dim), generator=gen).to(self.dt)
        T = self.total = sum(n for _, n in lens)
        self.cu = np.cumsum([0] + [n for _, n in lens])
        self.q = torch.randn((layers, T, hq, dim), generator=gen).to(self.dt)
        self.k = torch.randn((layers, T, hkv, dim), generator=gen).to(self.dt)
        self.v = torch.randn((layers, T, hkv, dim), generator=gen).to(self.dt)
        self.scale = float(np.float32(1) / np.sqrt(np.float32(dim)))

    def requests(self):
        return [cb.make_window_request(t, c, n, r) for r, ((c, n), t) in enumerate(zip(self.lens, self.tables))]

    def create(self, pool, stream=None):
        return cb.calvo_create(self.layers, self.hq, self.hkv, self.dim, cb.CALVO_BF16 if self.dtype == "bf16" else cb.CALVO_F32, self.slots, pool,
                               compute_stream=stream)

    def pool64(self, layer=0):
        """The pool as the oracle sees it, with the new tokens in place."""
        pool = self.pool[layer].double().numpy().copy()
        for r, ((c, n), t) in enumerate(zip(self.lens, self.tables)):
            a = self.cu[r]
            wo.append(pool, t, c, self.k[layer, a:a + n].double().numpy(), self.v[layer, a:a + n].double().numpy())
        return pool

    def stride(self, more=3):
        return max([c + n for c, n in self.lens] + [1]) + more

    def run(self, window, n_first=0, mass=False, last_rows=0, mass_in=None, scale=0.0, in_place=False):
        """Every layer once.  Returns a dict of CPU tensors."""
        dev = "cuda:0"
        pool, q, k, v = (x.to(dev) for x in (self.pool, self.q, self.k, self.v))
        guard = 8                                              # rows behind the last one: left as they are
        out = torch.full((self.layers, self.total + guard, self.hq, self.dim), 7.0, dtype=self.dt, device=dev)
        lse = torch.full((self.layers, self.total + guard, self.hq), 7.0, device=dev)
        rows, stride = len(self.lens) + 1, self.stride()
        got = torch.full((self.layers, rows, self.hkv, stride), -5.0, device=dev)
        given = None if mass_in is None else mass_in.to(dev)
        if in_place:
            got, given = given, given
        torch.cuda.synchronize()
        ctx = self.create(pool)
        try:
            plan = cb.calvo_window_prepare(ctx, self.requests(), window, n_first)
            for l in range(self.layers):
                cb.calvo_window_attn(plan, l, q[l], k[l], v[l], out[l], lse[l], scale)
                if mass:
                    cb.calvo_attn_mass(plan, l, q[l], lse[l], None if given is None else given[l], got[l], rows, stride, last_rows, scale)
            cb.calvo_window_destroy(plan)
        finally:
            cb.calvo_destroy(ctx)
        torch.cuda.synchronize()
        assert torch.equal(out[:, self.total:].float(), torch.full_like(out[:, self.total:], 7.0).float())
        assert torch.equal(lse[:, self.total:], torch.full_like(lse[:, self.total:], 7.0))
        return {"out": out[:, :self.total].cpu(), "lse": lse[:, :self.total].cpu(), "mass": got.cpu(), "pool": pool.cpu()}


def score_error(reach, dim):
    """Bound on the error of scale * <q, k> in fp32: dim products and sums of terms that add up to at most `reach`, each rounded, and the
    change of base of the exponential (three roundings of values up to reach)."""
    return (2 * dim + 8) * U32 * reach


def check_attn(c, got, window, n_first=0, layer=0, weight_step=0.0, scale=None, rows=None):
    """Every element within its bound: the error of a weight is that of its score, doubled by the division, and the sum over the keys
    adds half a step of fp32 per term; the output's rounding; weight_step: half a step of the type that weights are rounded to.
    rows: which new tokens of a request count (None: all)."""
    pool = c.pool64(layer)
    scale = c.scale if scale is None else scale
    for r, ((n_cached, n), t) in enumerate(zip(c.lens, c.tables)):
        if n == 0:
            continue
        a = int(c.cu[r])
        out, lse, mag, reach = wo.attn(pool, c.q[layer, a:a + n].double().numpy(), t, n_cached, n, window, n_first, scale)
        keys = min(n_cached + n, window + n_first)
        ds = score_error(reach, c.dim)
        g_out, g_lse = got["out"][layer, a:a + n].double().numpy(), got["lse"][layer, a:a + n].double().numpy()
        if rows is not None:
            out, lse, mag, reach, ds, g_out, g_lse = (x[rows] for x in (out, lse, mag, reach, ds, g_out, g_lse))
        tol = mag * (2 * ds[..., None] + (2 * keys + 64) * U32 + weight_step) + OUT[c.dtype] * (np.abs(out) + mag * 2 ** -7) + 1e-30
        bad = np.argwhere(~(np.abs(g_out - out) <= tol))
        assert len(bad) == 0, f"request {r}: {len(bad)} outputs, first {bad[0].tolist()}: {g_out[tuple(bad[0])]} for {out[tuple(bad[0])]} +- {tol[tuple(bad[0])]}"
        tol = ds + (2 * keys + 64) * U32 + 8 * U32 * (np.abs(lse) + reach)
        bad = np.argwhere(~(np.abs(g_lse - lse) <= tol))
        assert len(bad) == 0, f"request {r}: {len(bad)} lse, first {bad[0].tolist()}: {g_lse[tuple(bad[0])]} for {lse[tuple(bad[0])]}"


def check_pool(c, got):
    """The new tokens are in place, every other byte is as it was."""
    want = c.pool.clone()
    for r, ((n_cached, n), t) in enumerate(zip(c.lens, c.tables)):
        for i in range(n):
            p = n_cached + i
            want[:, t[p // B], 0, p % B] = c.k[:, c.cu[r] + i]
            want[:, t[p // B], 1, p % B] = c.v[:, c.cu[r] + i]
    as_int = torch.int16 if c.dtype == "bf16" else torch.int32
    assert torch.equal(got["pool"].view(as_int), want.view(as_int))


def check_mass(c, got, window, n_first=0, last_rows=0, mass_in=None, layer=0, scale=None, left=-5.0):
    """Against the definition with the log-sum-exp that the call was given."""
    pool = c.pool64(layer)
    scale = c.scale if scale is None else scale
    want_left = torch.full_like(got["mass"][layer], left) if mass_in is None or left is not None else mass_in[layer].clone()
    for r, ((n_cached, n), t) in enumerate(zip(c.lens, c.tables)):
        a = int(c.cu[r])
        q, lse = c.q[layer, a:a + n].double().numpy(), got["lse"][layer, a:a + n].double().numpy()
        before = None if mass_in is None else mass_in[layer, r].double().numpy()
        want = wo.mass(pool, q, lse, t, n_cached, n, window, n_first, scale, before, last_rows)
        k, _ = wo.tokens_of(pool, t, n_cached + n)
        reach = float(scale * np.abs(np.nan_to_num(q)).sum(-1).max() * np.abs(np.nan_to_num(k)).max()) if n else 0.0
        big = float(np.abs(lse).max()) if n else 0.0
        group = c.hq // c.hkv
        tol = np.abs(want) * (score_error(reach, c.dim) + 8 * U32 * big + (2 * n * group + 64) * U32) + 1e-35
        g = got["mass"][layer, r, :, :n_cached + n].double().numpy()
        bad = np.argwhere(~(np.abs(g - want) <= tol))
        assert len(bad) == 0, f"request {r}: {len(bad)} weights, first {bad[0].tolist()}: {g[tuple(bad[0])]} for {want[tuple(bad[0])]}"
        want_left[r, :, :n_cached + n] = got["mass"][layer, r, :, :n_cached + n]
    assert torch.equal(got["mass"][layer], want_left), "written outside the requests' tokens"
