"""A pool of 8-bit floats with a power of two as scale for each block, K or V, and head; the rotation of Q and K by position.  From their definitions in
numpy fp64 (test infrastructure only).

A block: K [Hkv][16][D] bytes, V [Hkv][D][16] bytes, scales fp32 [K, V][Hkv], up to a multiple of 128 bytes."""
import numpy as np

B = 16


def _values():
    """The number that each byte stands for: a sign, four bits of exponent (bias 7), three of fraction; 0x7f and 0xff are NaN."""
    out = np.zeros(256)
    for b in range(256):
        e, f = b >> 3 & 15, b & 7
        x = f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        out[b] = np.nan if b & 127 == 127 else -x if b >> 7 else x
    return out


VALUES = _values()


def decode(b):
    return VALUES[b]


def encode(x):
    """The byte of the nearest value, ties to the even one; |x| <= 448."""
    x = np.asarray(x, np.float64)
    mags = VALUES[:127]
    i = np.clip(np.searchsorted(mags, np.abs(x)), 1, 126)
    lo, hi = mags[i - 1], mags[i]
    up = (np.abs(x) - lo > hi - np.abs(x)) | ((np.abs(x) - lo == hi - np.abs(x)) & (i % 2 == 0))
    return (np.where(up, i, i - 1) | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def block_bytes(hkv, dim):
    return -(-(2 * hkv * B * dim + 8 * hkv) // 128) * 128


def parts(pool, hkv, dim):
    """Views of [slots][block bytes] uint8: K [slots][Hkv][16][D], V [slots][Hkv][D][16], scales [slots][2][Hkv]."""
    n = hkv * B * dim
    s = len(pool)
    return (pool[:, :n].reshape(s, hkv, B, dim), pool[:, n:2 * n].reshape(s, hkv, dim, B),
            np.ascontiguousarray(pool[:, 2 * n:2 * n + 8 * hkv]).view(np.float32).reshape(s, 2, hkv))


def widened(pool, hkv, dim):
    """[slots][2][16][Hkv][D] fp64, what the blocks stand for."""
    k, v, scale = parts(pool, hkv, dim)
    scale = scale.astype(np.float64)
    scale = np.where(np.isfinite(scale), scale, np.nan)
    with np.errstate(invalid="ignore"):
        k = decode(k) * scale[:, 0, :, None, None]
        v = decode(v) * scale[:, 1, :, None, None]
    return np.stack([k.transpose(0, 2, 1, 3), v.transpose(0, 3, 1, 2)], axis=1)


def least_scale(top):
    """The smallest power of two with top <= 448 times it (at least 2^-126)."""
    if not np.isfinite(top):
        return np.nan
    s = 2.0 ** -126
    while top > 448 * s:
        s *= 2
    return s


def rotate(x, pos, inv_freq, rot, interleaved):
    """x [tokens][heads][D], pos [tokens]."""
    y = np.array(x, np.float64)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        t = np.asarray(pos, np.float64) * float(inv_freq[i])
        co, si = np.cos(t)[:, None], np.sin(t)[:, None]
        y[..., a], y[..., b] = x[..., a] * co - x[..., b] * si, x[..., b] * co + x[..., a] * si
    return y


def append_block(held, scale, first, x):
    """One block and head: held [16][D] bytes, scale the one it has, x [n][D] the new values at tokens first ...  Returns (bytes of the tokens in front,
    values of the new ones over the new scale, not rounded, the new scale)."""
    s = least_scale(np.abs(x).max()) if np.isfinite(x).all() else np.nan
    if first:
        s = max(s, scale) if np.isfinite(s) and np.isfinite(scale) else np.nan
    if np.isnan(s):
        return np.zeros_like(held[:first]), np.zeros_like(x), s
    before = held[:first] if not first or s == scale else encode(decode(held[:first]) * (float(scale) / s))
    return before, x / s, s
