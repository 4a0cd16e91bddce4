"""Window attention, gathered weights and eviction on a paged pool, from their definitions in numpy fp64 (test infrastructure only).

pool: one layer, [slots][2][16][Hkv][D] in fp64.  A request is (table, n_cached, n_new); q: [new tokens][Hq][D]."""
import numpy as np

B = 16


def tokens_of(pool, table, n):
    """K and V of the first n tokens, [n][Hkv][D] each."""
    table = np.asarray(table, np.int64)
    pos = np.arange(n)
    return pool[table[pos // B], 0, pos % B], pool[table[pos // B], 1, pos % B]


def sees(pos, t, window, n_first):
    """Which of the positions t the rows at pos see, [rows][keys]."""
    p, t = np.asarray(pos, np.int64)[:, None], np.asarray(t, np.int64)[None, :]
    return (t <= p) & ((t > p - window) | (t < n_first))


def append(pool, table, n_cached, k_new, v_new):
    for i in range(len(k_new)):
        p = n_cached + i
        pool[table[p // B], 0, p % B] = k_new[i]
        pool[table[p // B], 1, p % B] = v_new[i]


def attn(pool, q, table, n_cached, n_new, window, n_first, scale):
    """out [n_new][Hq][D], lse [n_new][Hq], and for tolerances the sums of weight times |V| and, per row and head, of the largest
    scale * sum |q k|."""
    k, v = tokens_of(pool, table, n_cached + n_new)
    n, hq, d = q.shape
    g = hq // k.shape[1]
    seen = sees(np.arange(n_cached, n_cached + n_new), np.arange(n_cached + n_new), window, n_first)
    out, mag = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, reach = np.zeros((n, hq)), np.zeros((n, hq))
    for h in range(hq):
        kh, vh = k[:, h // g], v[:, h // g]
        for i in range(n):
            # only what the row sees takes part, whatever the rest holds
            ki, vi = kh[seen[i]], vh[seen[i]]
            s = scale * (ki @ q[i, h])
            top = s.max()
            w = np.exp(s - top)
            lse[i, h] = top + np.log(w.sum())
            w /= w.sum()
            out[i, h] = w @ vi
            mag[i, h] = w @ np.abs(vi)
            reach[i, h] = scale * (np.abs(ki) @ np.abs(q[i, h])).max()
    return out, lse, mag, reach


def mass(pool, q, lse, table, n_cached, n_new, window, n_first, scale, mass_in=None, last_rows=0):
    """[Hkv][n_cached + n_new] gathered weights; mass_in: [Hkv][>= n_cached]."""
    total = n_cached + n_new
    k, _ = tokens_of(pool, table, total)
    hkv = k.shape[1]
    g = q.shape[1] // hkv
    got = np.zeros((hkv, total))
    if mass_in is not None:
        got[:, :n_cached] = mass_in[:, :n_cached]
    seen = sees(np.arange(n_cached, total), np.arange(total), window, n_first)
    for i in range(max(0, n_new - last_rows) if last_rows else 0, n_new):
        for h in range(q.shape[1]):
            t = np.flatnonzero(seen[i])
            got[h // g, t] += np.exp(scale * (k[t, h // g] @ q[i, h]) - lse[i, h])
    return got


def choose(mass_row, n_tokens, n_keep, n_first, n_last):
    """Positions that stay, ascending."""
    def order(t):
        safe = t < n_first or t >= n_tokens - n_last
        x = float(mass_row[t])
        return (not safe, np.isnan(x), 0.0 if np.isnan(x) else -x, t)
    return np.array(sorted(sorted(range(n_tokens), key=order)[:n_keep]), np.int64)
