"""Test-side driver of the append with rotation and of pools of 8-bit floats.  Bytes of the pool that no cached token has are 0xff: NaN, as is a scale of
such bytes."""
import numpy as np
import torch

from oracle import e4m3_oracle as eo
from paper_2603_21257_amd import binding as cb
from window_harness import U32

B = 16
HALF_STEP = 2.0 ** -4                  # of an 8-bit float, relative; 2^-10 below 2^-6


class Case8:
    """Layers of an 8-bit pool, requests of (n_cached, n_new) tokens, q and the new K and V, scales around `size`."""

    def __init__(self, lens, hq=8, hkv=2, dim=64, seed=1, spare=5, layers=1, size=0.0):
        rng = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.dim, self.layers, self.dtype, self.dt = lens, hq, hkv, dim, layers, "bf16", torch.bfloat16
        blocks = [-(-(c + n) // B) for c, n in lens]
        self.slots = sum(blocks) + spare
        perm = rng.permutation(self.slots).astype(np.int32)
        at = np.cumsum([0] + blocks)
        self.tables = [perm[a:b].copy() for a, b in zip(at[:-1], at[1:])]
        self.pool = np.full((layers, self.slots, eo.block_bytes(hkv, dim)), 255, np.uint8)
        n8 = hkv * B * dim
        for l in range(layers):
            k, v = self.pool[l, :, :n8].reshape(-1, hkv, B, dim), self.pool[l, :, n8:2 * n8].reshape(-1, hkv, dim, B)
            scale = np.full((self.slots, 2, hkv), np.nan, np.float32)
            for (c, _), t in zip(lens, self.tables):
                for b in range(-(-c // B)):
                    m = min(B, c - b * B)
                    k[t[b], :, :m] = eo.encode(np.clip(rng.standard_normal((hkv, m, dim)) * 60, -448, 448))
                    v[t[b], :, :, :m] = eo.encode(np.clip(rng.standard_normal((hkv, dim, m)) * 60, -448, 448))
                    scale[t[b]] = 2.0 ** (rng.integers(-7, -4, (2, hkv)) + size)
            self.pool[l, :, :n8], self.pool[l, :, n8:2 * n8] = k.reshape(self.slots, -1), v.reshape(self.slots, -1)
            self.pool[l, :, 2 * n8:2 * n8 + 8 * hkv] = scale.reshape(self.slots, -1).view(np.uint8)
        T = self.total = sum(n for _, n in lens)
        self.cu = np.cumsum([0] + [n for _, n in lens])
        gen = torch.Generator().manual_seed(seed)
        self.q = torch.randn((layers, T, hq, dim), generator=gen).to(self.dt)
        self.k = torch.randn((layers, T, hkv, dim), generator=gen).to(self.dt)
        self.v = torch.randn((layers, T, hkv, dim), generator=gen).to(self.dt)
        self.scale = float(np.float32(1) / np.sqrt(np.float32(dim)))

    def requests(self):
        return [cb.make_window_request(t, c, n, -1) for (c, n), t in zip(self.lens, self.tables)]

    def create(self, pool, stream=None, **kw):
        return cb.calvo_create(self.layers, self.hq, self.hkv, self.dim, cb.CALVO_E4M3, self.slots, pool, compute_stream=stream, **kw)

    def pool64(self, layer=0):
        """What check_attn of window_harness compares with: the blocks as the GPU left them."""
        return eo.widened(self.after[layer], self.hkv, self.dim)

    def positions(self):
        return np.concatenate([np.arange(c, c + n) for c, n in self.lens] + [np.zeros(0, np.int64)])

    def run(self, window, n_first=0, scale=0.0, append=True, rope=None, far=None):
        """Every layer once: the append (rope: (inv_freq, rot, interleaved); far: positions) and the attention of what it left.  CPU tensors."""
        dev, guard = "cuda:0", 8
        pool = torch.from_numpy(self.pool).to(dev)
        q, k, v = (x.to(dev) for x in (self.q, self.k, self.v))
        out = torch.full((self.layers, self.total + guard, self.hq, self.dim), 7.0, dtype=self.dt, device=dev)
        q_out = torch.full_like(out, 7.0)
        lse = torch.full((self.layers, self.total + guard, self.hq), 7.0, device=dev)
        r = None
        if rope:
            r = cb.make_rope(torch.from_numpy(rope[0]).to(dev), rope[1], rope[2], None if far is None else torch.from_numpy(far.astype(np.int32)).to(dev))
        torch.cuda.synchronize()
        ctx = self.create(pool)
        try:
            plan = cb.calvo_window_prepare(ctx, self.requests(), window, n_first)
            for l in range(self.layers):
                if rope:
                    cb.calvo_kv_append(plan, l, k[l], v[l], q[l], q_out[l], r)
                    cb.calvo_window_attn(plan, l, q_out[l], None, None, out[l], lse[l], scale)
                else:
                    cb.calvo_window_attn(plan, l, q[l], k[l] if append else None, v[l] if append else None, out[l], lse[l], scale)
            cb.calvo_window_destroy(plan)
        finally:
            cb.calvo_destroy(ctx)
        torch.cuda.synchronize()
        for x in (out, lse) + ((q_out,) if rope else ()):
            assert (x[:, self.total:].float() == 7.0).all(), "written behind the last row"
        self.after = pool.cpu().numpy()
        return {"out": out[:, :self.total].cpu(), "lse": lse[:, :self.total].cpu(), "q": q_out[:, :self.total].cpu(), "pool": self.after}


def rotation_error(x, pos, rot):
    """Per element, the error of a rotation in fp32 of exact inputs: the fraction of a turn rounded to fp32 (2^-25 of half a turn, times pi: 1.6 * 2^-24),
    cosine and sine within 4 units in the last place, two products and a sum; turns in 64 bits (position times 2^-52, in radians)."""
    big = np.abs(np.asarray(x, np.float64)).max(axis=-1, keepdims=True)
    return 2 * big * (12 * U32 + np.abs(np.asarray(pos, np.float64))[:, None, None] * 2.0 ** -51) if rot else 0 * big


def check_append8(c, got, rope=None, far=None):
    """Every byte of the pool: the touched blocks by the definition, all others as they were."""
    n8 = c.hkv * B * c.dim
    pos = c.positions() if far is None else far
    for l in range(c.layers):
        want, got_l = c.pool[l].copy(), got["pool"][l]
        gk, gv, gs = eo.parts(got_l, c.hkv, c.dim)
        ok, ov, osc = eo.parts(c.pool[l], c.hkv, c.dim)
        k64, v64 = c.k[l].double().numpy(), c.v[l].double().numpy()
        err = np.zeros(k64.shape[:1] + (1, 1))
        if rope:
            err = np.broadcast_to(rotation_error(k64, pos, rope[1]), k64.shape[:2] + (1,))
            k64 = eo.rotate(k64, pos, *rope)
        err = np.broadcast_to(err, k64.shape[:2] + (1,))
        for r, ((cached, n), t) in enumerate(zip(c.lens, c.tables)):
            for b in range(cached // B, -(-(cached + n) // B) if n else 0):
                lo, hi = max(cached, b * B), min(cached + n, b * B + B)
                a, e, s = lo - b * B, hi - b * B, t[b]
                rows = slice(c.cu[r] + lo - cached, c.cu[r] + hi - cached)
                for h in range(c.hkv):
                    for which, x in ((0, k64[rows, h]), (1, v64[rows, h])):
                        held = gk[s, h] if which == 0 else gv[s, h].T
                        old = ok[s, h] if which == 0 else ov[s, h].T
                        before, now, scale = eo.append_block(old, osc[s, which, h], a, x)
                        name = f"layer {l} request {r} block {b} head {h} {'KV'[which]}"
                        if np.isnan(scale):
                            assert np.isnan(gs[s, which, h]), name
                            continue
                        slack = err[rows, h] if which == 0 else np.zeros((hi - lo, 1))
                        if gs[s, which, h] != scale:             # the largest value may lie within its error of the border
                            top = np.abs(x).max() / 448
                            assert abs(np.log2(top) - np.round(np.log2(top))) < 1e-6, (name, gs[s, which, h], scale)
                            continue
                        assert np.array_equal(held[:a], before), name
                        assert (held[e:] == 0).all(), name
                        off = np.abs(eo.decode(held[a:e]) - now)
                        tol = np.maximum(HALF_STEP * np.abs(now), 2.0 ** -10) + 2 * slack / scale
                        assert (off <= tol).all(), (name, off.max())
                # compared above: not looked at below
                want[s] = got_l[s]
                want[s, 2 * n8 + 8 * c.hkv:] = c.pool[l, s, 2 * n8 + 8 * c.hkv:]
        assert np.array_equal(got_l, want), "written outside the touched blocks"


def check_q(c, got, rope, far=None, out=2.0 ** -8):
    pos = c.positions() if far is None else far
    for l in range(c.layers):
        x = c.q[l].double().numpy()
        want = eo.rotate(x, pos, *rope)
        off = np.abs(got["q"][l].double().numpy() - want)
        assert (off <= rotation_error(x, pos, rope[1]) * (1 + out) + out * np.abs(want) + 1e-38).all(), off.max()


def inv_freq(rot, base=10000.0):
    return (base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)).astype(np.float32)
