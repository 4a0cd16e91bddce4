"""The operators that keep a request's cache bounded, as cases: attention of new tokens with a sliding window and a few
first tokens that stay visible, the attention weight that every cached token has gathered, and the move of the tokens that have
gathered most into fewer slots.

A case's "op":
  "attn"   one step of a serving program: a plan for the batch (calvo_window_prepare), then for every layer the new tokens'
           K and V into the paged pool and their attention (calvo_window_attn), which also leaves the rows' log-sum-exp
  "mass"   one layer's gathered weights with those of the new tokens added (calvo_attn_mass)
  "evict"  the kept tokens of every layer and KV head, moved into the slots of a shorter table (calvo_kv_evict)
"lens" holds a request's lengths as "C+N" (cached and new tokens; "evict": "L-K", cached and kept tokens), requests separated
by commas.  "window" 0 stands for one that hides nothing.
"""
import math
import weakref

import numpy as np
import torch

own = False

B = 16                          # tokens of a block, the unit in which the pool is paged
NO_WINDOW = (1 << 31) - 1


def _case(name, op, lens, hq=32, hkv=8, dim=128, dtype="bf16", layers=1, window=0, sink=0, last_rows=0, first=0, last=0):
    c = {"op": op, "lens": lens, "hq": hq, "hkv": hkv, "dim": dim, "dtype": dtype, "layers": layers, "window": window, "sink": sink,
         "last_rows": last_rows, "first": first, "last": last}
    return dict({"name": name}, **c) if name else c


def listed():
    batch = ",".join("%d+1" % round(300 * 110 ** (i / 31)) for i in range(32))
    return [
        # one request that answers token by token behind a short window: the smallest step, launches and host time are what it costs
        _case("decode_one", "attn", "4096+1", layers=4, window=1024, sink=4),
        # a step of 32 requests of 300 to 33000 tokens, one new token each
        _case("decode_batch", "attn", batch, layers=2, window=4096, sink=64),
        # the three mean lengths of short queries over long contexts, as one ragged batch
        _case("queries_28k", "attn", "28096+28,28304+61,38304+209", window=8192, sink=4),
        # a chunk of a long prompt
        _case("chunk_16k_2k", "attn", "16384+2048", window=4096, sink=4),
        # a whole prompt in one call, the largest
        _case("prompt_32k", "attn", "0+32768", window=4096, sink=128),
        # 64-wide heads, a chunk that begins and ends inside a block, a window without first tokens
        _case("head64_chunk", "attn", "4111+300", hq=16, hkv=4, dim=64, window=2048),
        # fp32 pool, 64-wide heads, a window shorter than the chunk and its context
        _case("fp32_chunk", "attn", "1000+128", hq=8, hkv=2, dim=64, dtype="f32", window=300, sink=5),
        # one new token each of 8 requests, whose weights are added to what the cached tokens have gathered
        _case("mass_decode", "mass", "4096+1,6001+1,8192+1,10007+1,12000+1,14321+1,16384+1,20000+1"),
        # a short query that looks over a long context
        _case("mass_query_28k", "mass", "28096+28"),
        # a whole prompt's rows under the mask that its attention had
        _case("mass_prompt_8k", "mass", "0+8192"),
        # a small fp32 cache to a quarter, a ragged length
        _case("evict_2k", "evict", "2011-512", hq=8, hkv=2, dim=64, dtype="f32", layers=4, first=4, last=64),
        # all layers of a long context to an eighth
        _case("evict_16k", "evict", "16384-2048", layers=32, first=4, last=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: attention most often, then gathered weights and evictions.  Element type, head layout and width, batch size, lengths,
    window and first tokens are drawn."""
    while True:
        op = rng.choices(["attn", "mass", "evict"], [5, 3, 2])[0]
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        dim = rng.choice([128, 128, 128, 64, 64, 40, 80, 96, 256])
        hq, hkv = rng.choice([(32, 8), (32, 8), (40, 8), (64, 8), (16, 2), (16, 4), (8, 8), (6, 3)])
        n = rng.choice([1, 1, 2, 3, 8, 24])
        lens = []
        for _ in range(n):
            if op == "evict":
                tokens = _log_int(rng, 64, 65536)
                lens.append("%d-%d" % (tokens, rng.randint(1, tokens) if rng.random() < 0.3 else max(1, tokens // rng.randint(2, 16))))
            else:
                new = 1 if n > 3 or rng.random() < 0.3 else _log_int(rng, 2, 512) if rng.random() < 0.6 else _log_int(rng, 512, 8192)
                lens.append("%d+%d" % (rng.choice([0, 1, 1, 1, 1, 1]) * _log_int(rng, 16, 65536), new))
        window = 0 if rng.random() < (0.15 if op == "attn" else 0.6) else _log_int(rng, 16, 16384)
        c = _case(None, op, ",".join(lens), hq, hkv, dim, dtype, 1, window, rng.choice([0, 1, 4, 4, 16, 100, 256]) if window else 0)
        if op == "evict":
            least = min(k for _, k in _lens(c))
            c["first"], c["last"], c["window"], c["sink"] = min(4, least // 2), min(least // 4, 256), 0, 0
            c["layers"] = rng.randint(1, 8)
        if op == "attn":
            c["layers"] = rng.randint(1, 4) if n > 3 else 1
        if op == "mass" and rng.random() < 0.3:
            c["last_rows"] = rng.choice([1, 16, 64])
        # no dearer than the listed ones, in a pool that leaves room for others
        w, elt = work(c), 2 if dtype == "bf16" else 4
        tokens = sum(a + b for a, b in _lens(c))
        if w["flops"] <= 6e11 / (16 if dtype == "f32" else 1) and w["bytes"] <= 5.5e8 and 2 * tokens * hkv * dim * elt * c["layers"] <= 6e9:
            return c


# ---- inputs

def _lens(case):
    return [tuple(int(x) for x in ps.replace("-", "+").split("+")) for ps in case["lens"].split(",")]


def _tdtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _window(case):
    return case["window"] or NO_WINDOW


def _scale(case):
    return float(np.float32(1.0) / np.sqrt(np.float32(case["dim"])))


def _seen(case, c, n):
    """Where the keys begin that the rows of a request (c cached, n new tokens) see besides the first ones."""
    return max(0, c + 1 - _window(case))


def _mass_stride(case):
    return -(-max(a + (b if case["op"] != "evict" else 0) for a, b in _lens(case)) // 64) * 64


def _normal(shape, dtype, gen):
    return torch.empty(shape, dtype=dtype, device="cuda:0").normal_(generator=gen)


class _Handles:
    """Context and plan of one state; given back when the state goes."""

    def __init__(self, cb, ctx, plan, keep):
        self.ctx, self.plan = ctx, plan
        self._fin = weakref.finalize(self, _Handles._close, cb, ctx, plan, keep)

    @staticmethod
    def _close(cb, ctx, plan, keep):
        if plan:
            cb.calvo_window_destroy(plan)
        cb.calvo_destroy(ctx)
        del keep


def prepare(case, seed):
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    lens, dt = _lens(case), _tdtype(case)
    evict = case["op"] == "evict"
    L, hq, hkv, D = case["layers"], case["hq"], case["hkv"], case["dim"]
    blocks = [(-(-a // B), -(-b // B)) if evict else (-(-(a + b) // B), 0) for a, b in lens]
    need = sum(a + b for a, b in blocks)
    slots = need * 5 // 4 + 8
    perm = np.random.default_rng(seed).permutation(slots).astype(np.int32)
    tables, at = [], 0
    for a, b in blocks:
        tables.append((perm[at:at + a], perm[at + a:at + a + b]))
        at += a + b
    pool = _normal((L, slots, 2, B, hkv, D), dt, gen)
    st = {"case": case, "lens": lens, "pool": pool, "tables": tables,
          "index": [tuple(torch.from_numpy(t.astype(np.int64)).to("cuda:0") for t in ts) for ts in tables]}
    if evict:
        # gathered weights are skewed: a few tokens have most of them, some have none that fp32 holds
        stride = _mass_stride(case)
        mass = _normal((L, len(lens), hkv, stride), torch.float32, gen).mul_(2).exp_()
        mass[torch.rand(mass.shape, device="cuda:0", generator=gen) < 0.05] = 0
        keep = max(k for _, k in lens)
        st["mass"] = mass
        st["kept"] = torch.zeros((L, len(lens), hkv, keep), dtype=torch.int32, device="cuda:0")
        st["mass_out"] = torch.zeros((L, len(lens), hkv, keep), dtype=torch.float32, device="cuda:0")
    else:
        T = sum(n for _, n in lens)
        st["q"] = _normal((L, T, hq, D), dt, gen)
        st["lse"] = torch.zeros((L, T, hq), dtype=torch.float32, device="cuda:0")
        if case["op"] == "attn":
            st["k"] = _normal((L, T, hkv, D), dt, gen)
            st["v"] = _normal((L, T, hkv, D), dt, gen)
            st["out"] = torch.zeros((L, T, hq, D), dtype=dt, device="cuda:0")
        else:
            # what the layer's attention left: the rows' log-sum-exp; and what the cached tokens had gathered before
            stride = _mass_stride(case)
            _plain_attn(st, 0, with_out=False)
            st["mass_in"] = _normal((len(lens), hkv, stride), torch.float32, gen).exp_()
            st["mass_out"] = torch.zeros((len(lens), hkv, stride), dtype=torch.float32, device="cuda:0")
    torch.cuda.synchronize()
    if own:
        from paper_2603_21257_amd import binding as cb
        ctx = cb.calvo_create(L, hq, hkv, D, cb.CALVO_BF16 if case["dtype"] == "bf16" else cb.CALVO_F32, slots, pool)
        plan = None
        if evict:
            st["reqs"] = [cb.make_evict_request(src, a, dst, b, case["first"], case["last"], r)
                          for r, ((a, b), (src, dst)) in enumerate(zip(lens, tables))]
        else:
            st["reqs"] = [cb.make_window_request(t, c, n, r) for r, ((c, n), (t, _)) in enumerate(zip(lens, tables))]
            if case["op"] == "mass":                  # the plan of the step whose attention came before
                plan = cb.calvo_window_prepare(ctx, st["reqs"], _window(case), case["sink"])
        st["h"] = _Handles(cb, ctx, plan, [v for v in st.values() if isinstance(v, torch.Tensor)])
    return st


# ---- the plain form

def _plain_kv(st, l, r, n, which):
    """K (0) or V (1) of the first n tokens of request r, heads in front, in 32 bits."""
    x = st["pool"][l][st["index"][r][0], which]
    return x.reshape(-1, *x.shape[2:])[:n].permute(1, 0, 2).float().contiguous()


def _plain_rows(case, c, i, m):
    """Keys that rows i .. i + m - 1 of a request are measured against, and which of them each row sees."""
    window, sink, device = _window(case), case["sink"], "cuda:0"
    a = max(0, c + i + 1 - window)
    first = torch.arange(0, min(sink, a), device=device)
    keys = torch.cat([first, torch.arange(a, c + i + m, device=device)])
    pos = torch.arange(c + i, c + i + m, device=device)[:, None]
    return keys, (keys <= pos) & ((keys > pos - window) | (keys < sink))


def _plain_attn(st, l, with_out=True):
    case = st["case"]
    hq, hkv, D = case["hq"], case["hkv"], case["dim"]
    G, at, scale = hq // hkv, 0, _scale(case)
    for r, (c, n) in enumerate(st["lens"]):
        if with_out:                                   # the new tokens' K and V into the pool
            pos = torch.arange(c, c + n, device="cuda:0")
            slot = st["index"][r][0][pos // B]
            st["pool"][l][slot, 0, pos % B] = st["k"][l, at:at + n]
            st["pool"][l][slot, 1, pos % B] = st["v"][l, at:at + n]
        k = _plain_kv(st, l, r, c + n, 0)
        v = _plain_kv(st, l, r, c + n, 1) if with_out else None
        step = max(1, min(n, 1024, (1 << 28) // (hq * min(c + n, _window(case) + 1024 + case["sink"]))))
        for i in range(0, n, step):
            m = min(step, n - i)
            keys, sees = _plain_rows(case, c, i, m)
            q = st["q"][l, at + i:at + i + m].float().view(m, hkv, G, D).permute(1, 2, 0, 3).reshape(hkv, G * m, D)
            s = torch.matmul(q, k[:, keys].transpose(1, 2)).view(hkv, G, m, -1).mul_(scale)
            s.masked_fill_(~sees, -math.inf)
            top = s.amax(dim=-1, keepdim=True)
            w = s.sub_(top).exp_()
            total = w.sum(dim=-1, keepdim=True)
            st["lse"][l, at + i:at + i + m] = (top + total.log()).view(hkv * G, m).t()
            if with_out:
                o = torch.matmul(w.view(hkv, G * m, -1), v[:, keys]).view(hkv, G, m, D) / total
                st["out"][l, at + i:at + i + m] = o.permute(2, 0, 1, 3).reshape(m, hq, D).to(st["out"].dtype)
        at += n


def _plain_mass(st):
    case = st["case"]
    hq, hkv, D = case["hq"], case["hkv"], case["dim"]
    G, at, scale = hq // hkv, 0, _scale(case)
    for r, (c, n) in enumerate(st["lens"]):
        k = _plain_kv(st, 0, r, c + n, 0)
        total = torch.zeros((hkv, c + n), dtype=torch.float64, device="cuda:0")
        total[:, :c] = st["mass_in"][r, :, :c]
        i0 = max(0, n - case["last_rows"]) if case["last_rows"] else 0
        step = max(1, min(n, 1024, (1 << 27) // (hq * min(c + n, _window(case) + 1024 + case["sink"]))))
        for i in range(i0, n, step):
            m = min(step, n - i)
            keys, sees = _plain_rows(case, c, i, m)
            q = st["q"][0, at + i:at + i + m].float().view(m, hkv, G, D).permute(1, 2, 0, 3).reshape(hkv, G * m, D)
            s = torch.matmul(q, k[:, keys].transpose(1, 2)).view(hkv, G, m, -1).mul_(scale)
            s -= st["lse"][0, at + i:at + i + m].t().reshape(hkv, G, m, 1)
            total[:, keys] += s.masked_fill_(~sees, -math.inf).exp_().sum(dim=(1, 2), dtype=torch.float64)
        st["mass_out"][r, :, :c + n] = total.float()
        at += n


def _plain_evict(st):
    case, dev = st["case"], "cuda:0"
    for r, (tokens, keep) in enumerate(st["lens"]):
        src, dst = st["index"][r]
        rank = st["mass"][:, r, :, :tokens].clone()
        rank[..., :case["first"]] = math.inf
        rank[..., tokens - case["last"]:] = math.inf
        best = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :keep]
        kept = torch.sort(best, dim=-1)[0]                                     # [layers][hkv][keep], ascending
        st["kept"][:, r, :, :keep] = kept
        st["mass_out"][:, r, :, :keep] = st["mass"][:, r].gather(2, kept)
        head = torch.arange(case["hkv"], device=dev)[:, None]
        j = torch.arange(keep, device=dev)
        for l in range(case["layers"]):
            for which in (0, 1):
                rows = st["pool"][l][src[kept[l] // B], which, kept[l] % B, head]          # [hkv][keep][D]
                st["pool"][l][dst[j // B][None], which, (j % B)[None], head] = rows


# ---- one pass

def run(st):
    case = st["case"]
    if own:
        from paper_2603_21257_amd import binding as cb
        h = st["h"]
        if case["op"] == "attn":
            plan = cb.calvo_window_prepare(h.ctx, st["reqs"], _window(case), case["sink"])
            for l in range(case["layers"]):
                cb.calvo_window_attn(plan, l, st["q"][l], st["k"][l], st["v"][l], st["out"][l], st["lse"][l])
            cb.calvo_window_destroy(plan)
        elif case["op"] == "mass":
            cb.calvo_attn_mass(h.plan, 0, st["q"][0], st["lse"][0], st["mass_in"], st["mass_out"], len(st["lens"]), _mass_stride(case),
                               case["last_rows"])
        else:
            cb.calvo_kv_evict(h.ctx, st["reqs"], 0, case["layers"], st["mass"], len(st["lens"]), _mass_stride(case), st["kept"],
                              st["kept"].shape[-1], st["mass_out"], st["mass_out"].shape[-1])
    elif case["op"] == "attn":
        for l in range(case["layers"]):
            _plain_attn(st, l)
    elif case["op"] == "mass":
        _plain_mass(st)
    else:
        _plain_evict(st)
    if case["op"] == "attn":
        return {"out": st["out"], "lse": st["lse"], "pool": st["pool"]}
    if case["op"] == "mass":
        return {"mass": st["mass_out"]}
    return {"kept": st["kept"], "mass": st["mass_out"], "pool": st["pool"]}


# ---- what a pass cannot do without

def work(case):
    elt = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, D, L = case["hq"], case["hkv"], case["dim"], case["layers"]
    nbytes = flops = 0
    for a, b in _lens(case):
        if case["op"] == "evict":
            # gathered weights read; the kept rows of K and V read and written, their places and weights written
            nbytes += hkv * (4 * a + 4 * b * D * elt + 8 * b)
            continue
        c, n = a, b
        if case["last_rows"]:
            c, n = a + max(0, b - case["last_rows"]), min(b, case["last_rows"])
        lo = _seen(case, c, n)
        keys = c + n - lo + min(case["sink"], lo)
        p = np.arange(c, c + n, dtype=np.int64) + 1
        pairs = int(np.minimum(p, _window(case)).sum() + np.clip(p - _window(case), 0, case["sink"]).sum())
        if case["op"] == "attn":
            # K and V that some row sees (the new ones from the caller's arrays) read, the new ones stored; q read, out and lse written
            nbytes += 2 * hkv * D * elt * (keys + n) + n * hq * (2 * D * elt + 4)
            flops += 4 * D * hq * pairs
        else:
            # K, q and lse read; gathered weights read where there are cached tokens, and written
            nbytes += hkv * D * elt * keys + n * hq * (D * elt + 4) + 4 * hkv * (a + a + b)
            flops += 2 * D * hq * pairs
    return {"bytes": nbytes * L, "flops": flops * L}


# ---- the definition, in 64 bits

def _exact_cached(st, l, r, n, which, g):
    slots = st["index"][r][0]
    pos = torch.arange(n, device="cuda:0")
    return st["pool"][l, slots[pos // B], which, pos % B, g].double()


def exact(case, seed):
    st = prepare_inputs(case, seed)
    lens, hq, hkv, D = st["lens"], case["hq"], case["hkv"], case["dim"]
    G, W, sink = hq // hkv, _window(case), case["sink"]
    scale = _scale(case)
    if case["op"] == "evict":
        kept, mass = st["kept"].clone(), st["mass_out"].double()
        for r, (tokens, keep) in enumerate(lens):
            safe = torch.zeros(tokens, dtype=torch.bool, device="cuda:0")
            safe[:case["first"]] = True
            safe[tokens - case["last"]:] = True
            for l in range(case["layers"]):
                for g in range(hkv):
                    x = st["mass"][l, r, g, :tokens].double()
                    # a token's place in the order: protected first, then by weight, then by position
                    order = np.lexsort((np.arange(tokens), -x.cpu().numpy(), (~safe).cpu().numpy()))
                    at = torch.from_numpy(np.sort(order[:keep])).to("cuda:0")
                    kept[l, r, g, :keep] = at
                    mass[l, r, g, :keep] = x[at]
        return {"kept": kept, "mass": mass, "pool": None}
    T = sum(n for _, n in lens)
    out = torch.zeros((case["layers"], T, hq, D), dtype=torch.float64, device="cuda:0") if case["op"] == "attn" else None
    lse = torch.zeros((case["layers"], T, hq), dtype=torch.float64, device="cuda:0")
    gathered = st["mass_out"].double() if case["op"] == "mass" else None
    for l in range(case["layers"]):
        at = 0
        for r, (c, n) in enumerate(lens):
            for g in range(hkv):
                k = _exact_cached(st, l, r, c + n, 0, g)
                v = _exact_cached(st, l, r, c + n, 1, g) if out is not None else None
                if out is not None:
                    k[c:], v[c:] = st["k"][l, at:at + n, g].double(), st["v"][l, at:at + n, g].double()
                else:
                    gathered[r, g, :c], gathered[r, g, c:c + n] = st["mass_in"][r, g, :c].double(), 0
                rows = max(1, min(n, 512, (1 << 26) // (c + n)))
                for i in range(0, n, rows):
                    m = min(rows, n - i)
                    # without first tokens keys in front of every row's window are left out
                    lo = 0 if sink else max(0, c + i + 1 - W)
                    t = torch.arange(lo, c + i + m, device="cuda:0")[None, :]
                    p = torch.arange(c + i, c + i + m, device="cuda:0")[:, None]
                    hidden = (t > p) | ((t <= p - W) & (t >= sink))
                    kt = k[lo:c + i + m].t().contiguous()
                    for h in range(g * G, (g + 1) * G):
                        x = torch.matmul(st["q"][l, at + i:at + i + m, h].double(), kt) * scale
                        x[hidden] = -math.inf
                        z = torch.logsumexp(x, dim=1)
                        lse[l, at + i:at + i + m, h] = z
                        if out is not None:
                            out[l, at + i:at + i + m, h] = torch.matmul(torch.exp(x - z[:, None]), v[lo:c + i + m])
                        else:
                            # the weights are those of the log-sum-exp that was passed, rounded as it is
                            wgt = torch.exp(x - st["lse"][l, at + i:at + i + m, h].double()[:, None])
                            if case["last_rows"]:
                                wgt = wgt[max(0, n - case["last_rows"] - i):]
                            gathered[r, g, lo:c + i + m] += wgt.sum(dim=0)
            at += n
    if case["op"] == "attn":
        return {"out": out, "lse": lse, "pool": None}
    return {"mass": gathered}


def prepare_inputs(case, seed):
    """The inputs of prepare alone."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
