"""The append with rotation and 8-bit pools as a program uses them: contexts loaded from host memory, prompts in chunks and single tokens over the pool's own
allocator, captured graphs, plans and streams in turn, pools of more than 4 GiB, and refusals that write nothing."""
import numpy as np
import pytest
import torch

import e4m3_harness as eh
import window_harness as wh
from e4m3_harness import Case8, inv_freq
from oracle import e4m3_oracle as eo
from oracle import window_oracle as wo
from paper_2603_21257_amd import binding as cb
from window_harness import FULL, Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def buffers(c):
    """Device copies of a case's arrays: pool, q, k, v, q_out, out, lse."""
    pool = (torch.from_numpy(c.pool) if isinstance(c.pool, np.ndarray) else c.pool).to(DEV)
    q, k, v = c.q.to(DEV), c.k.to(DEV), c.v.to(DEV)
    torch.cuda.synchronize()
    return pool, q, k, v, torch.zeros_like(q), torch.zeros_like(q), torch.zeros((c.layers, c.total, c.hq), device=DEV)


@pytest.mark.parametrize("how", ["staged", "zero copy", "chunked", "remote"])
def test_contexts_loaded_from_host_memory(how):
    """Blocks of 8 bits through the loading stages, with the append and the attention queued behind them while they are under way."""
    L, hq, hkv, D, blocks, n = 3, 8, 2, 128, 24, 20
    c = Case8([(16 * blocks, n)], hq, hkv, D, seed=3, layers=L)
    nbytes = cb.calvo_block_bytes(hkv, D, cb.CALVO_E4M3)
    t = c.tables[0]
    host = torch.from_numpy(np.ascontiguousarray(c.pool[:, t[:blocks]]))
    if how != "remote":
        host = torch.empty_like(host, pin_memory=True).copy_(host)
    want = c.run(FULL, rope=(inv_freq(D), D, False))
    rope = cb.make_rope(torch.from_numpy(inv_freq(D)).to(DEV), D)
    pool, q, k, v, q_out, out, lse = buffers(c)
    pool.fill_(255)
    torch.cuda.synchronize()
    ctx = c.create(pool, staging_bytes=0 if how == "zero copy" else 8 * nbytes)
    req = [cb.make_request(host, blocks * nbytes, t, blocks, n)]
    if how == "chunked":
        cb.calvo_kv_ingest_chunked(ctx, req, 0, L, [4, 0, 8])
    elif how == "remote":
        cb.calvo_kv_ingest_l3(ctx, req, 0, L, chunk_bytes=4 * nbytes, l3_GBps=2.0)
    else:
        cb.calvo_kv_ingest(ctx, req, 0, L)
    plan = cb.calvo_window_prepare(ctx, c.requests(), FULL)
    for l in range(L):
        cb.calvo_kv_append(plan, l, k[l], v[l], q[l], q_out[l], rope)
        cb.calvo_window_attn(plan, l, q_out[l], None, None, out[l], lse[l])
    if how == "remote":
        cb.calvo_l3_wait(ctx)
    cb.calvo_window_destroy(plan)
    cb.calvo_destroy(ctx)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu(), want["out"]) and torch.equal(lse.cpu(), want["lse"])
    used = np.sort(t)
    assert np.array_equal(pool.cpu().numpy()[:, used, :2 * hkv * 16 * D], want["pool"][:, used, :2 * hkv * 16 * D])


@pytest.mark.parametrize("hq,hkv,dim,window,n_first", [(8, 2, 128, FULL, 0), (8, 2, 64, 60, 3), (32, 8, 128, 100, 20)])
def test_a_request_from_prompt_to_tokens(hq, hkv, dim, window, n_first):
    """Two layers, a prompt in two chunks, then single tokens, rotated by position: every step by the definition on what the GPU held before it."""
    L, slots = 2, 30
    gen = torch.Generator().manual_seed(4)
    pool = torch.full((L, slots, eo.block_bytes(hkv, dim)), 255, dtype=torch.uint8, device=DEV)
    f = inv_freq(dim)
    rope = cb.make_rope(torch.from_numpy(f).to(DEV), dim)
    ctx = cb.calvo_create(L, hq, hkv, dim, cb.CALVO_E4M3, slots, pool)
    alloc = cb.calvo_pool_create(slots)
    table, cached = np.zeros(0, np.int32), 0
    for n in (37, 90, 1, 1, 1, 17, 1):
        more = -(-(cached + n) // 16) - len(table)
        if more:
            table = np.concatenate([table, cb.calvo_pool_reserve(alloc, more)])
        c = Case8([(0, n)], hq, hkv, dim, layers=L, spare=slots)
        c.lens, c.tables, c.slots, c.pool = [(cached, n)], [table], slots, pool.cpu().numpy()
        c.q, c.k, c.v = (torch.randn((L, n, h, dim), generator=gen).to(c.dt) for h in (hq, hkv, hkv))
        _, q, k, v, q_out, out, lse = buffers(c)
        plan = cb.calvo_window_prepare(ctx, c.requests(), window, n_first)
        for l in range(L):
            cb.calvo_kv_append(plan, l, k[l], v[l], q[l], q_out[l], rope)
            cb.calvo_window_attn(plan, l, q_out[l], None, None, out[l], lse[l])
        cb.calvo_window_destroy(plan)
        torch.cuda.synchronize()
        got = {"pool": pool.cpu().numpy(), "q": q_out.cpu(), "out": out.cpu(), "lse": lse.cpu()}
        eh.check_append8(c, got, (f, dim, False))
        eh.check_q(c, got, (f, dim, False))
        c.after, c.q = got["pool"], got["q"]
        for l in range(L):
            wh.check_attn(c, got, window, n_first, l, 2.0 ** -8)
        cached += n
    cb.calvo_destroy(ctx)
    cb.calvo_pool_destroy(alloc)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_wide_pools_append_then_attend(dtype, dim):
    """Rotated by the append, then attention: the same bits as attention that stores the rotated K itself."""
    c = Case([(100, 1), (0, 33), (257, 70)], 8, 2, dim, dtype, seed=5)
    pool, q, k, v, q_out, out, lse = buffers(c)
    other = pool.clone()
    rope = cb.make_rope(torch.from_numpy(inv_freq(dim)).to(DEV), dim)
    torch.cuda.synchronize()
    ctx = c.create(pool)
    plan = cb.calvo_window_prepare(ctx, c.requests(), 90, 4)
    cb.calvo_kv_append(plan, 0, k[0], v[0], q[0], q_out[0], rope)
    cb.calvo_window_attn(plan, 0, q_out[0], None, None, out[0], lse[0])
    cb.calvo_window_destroy(plan)
    cb.calvo_destroy(ctx)
    rotated = torch.empty_like(k)
    for (a, n), t, at in zip(c.lens, c.tables, c.cu):
        for i in range(n):
            rotated[0, at + i] = pool[0, t[(a + i) // 16], 0, (a + i) % 16]
    out2, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    torch.cuda.synchronize()
    ctx = c.create(other)
    plan = cb.calvo_window_prepare(ctx, c.requests(), 90, 4)
    cb.calvo_window_attn(plan, 0, q_out[0], rotated[0], v[0], out2[0], lse2[0])
    cb.calvo_window_destroy(plan)
    cb.calvo_destroy(ctx)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    assert torch.equal(pool.nan_to_num(5.0), other.nan_to_num(5.0))


def test_attention_appends_as_the_append_does():
    c = Case8([(20, 3), (33, 50), (0, 1)], 8, 2, 128, seed=6, layers=2)
    a = c.run(FULL)
    pool, q, k, v, _, out, lse = buffers(c)
    ctx = c.create(pool)
    plan = cb.calvo_window_prepare(ctx, c.requests(), FULL)
    for l in range(2):
        cb.calvo_kv_append(plan, l, k[l], v[l])
        cb.calvo_window_attn(plan, l, q[l], None, None, out[l], lse[l])
        cb.calvo_window_attn(plan, l, q[l], None, None, out[l], lse[l])          # the same call gives the same bits
    cb.calvo_window_destroy(plan)
    cb.calvo_destroy(ctx)
    assert torch.equal(out.cpu(), a["out"]) and torch.equal(lse.cpu(), a["lse"]) and np.array_equal(pool.cpu().numpy(), a["pool"])


def test_q_copied_and_parts_of_fused_rows():
    """Strides: q, k and v as parts of the rows of one array, with room behind; q without a rope is copied."""
    c = Case8([(9, 30)], 8, 2, 64, seed=7)
    want = c.run(FULL, rope=(inv_freq(64), 64, True))
    row = (8 + 2 + 2) * 64 + 24
    rows = torch.full((c.total, row), float("nan"), dtype=torch.bfloat16)
    rows[:, :512], rows[:, 512:640], rows[:, 648:776] = (x[0].reshape(c.total, -1) for x in (c.q, c.k, c.v))
    rows = rows.to(DEV)
    pool, q, k, v, q_out, out, lse = buffers(c)
    rope = cb.make_rope(torch.from_numpy(inv_freq(64)).to(DEV), 64, True)
    ctx = c.create(pool)
    plan = cb.calvo_window_prepare(ctx, c.requests(), FULL)
    at = rows.data_ptr()
    cb.calvo_kv_append(plan, 0, at + 2 * 512, at + 2 * 648, at, q_out[0], rope, row, row, row)
    copied = torch.zeros_like(q_out[0])
    cb.calvo_kv_append(plan, 0, None, None, at, copied, None, 0, 0, row)
    cb.calvo_window_destroy(plan)
    cb.calvo_destroy(ctx)
    assert np.array_equal(pool.cpu().numpy(), want["pool"]) and torch.equal(q_out.cpu(), want["q"]) and torch.equal(copied.cpu(), c.q[0])


@pytest.mark.parametrize("lens", [[(300, 1), (75, 1)], [(200, 60)]])
@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_captured(lens, kind):
    """Two plans, each step captured, replayed in turn with eager work between them; every replay against the eager result."""
    cases = [(Case8 if kind == "e4m3" else Case)(lens, 8, 2, 128, seed=s) for s in (41, 42)]
    side = torch.cuda.Stream()
    f = torch.from_numpy(inv_freq(128)).to(DEV)
    rope = cb.make_rope(f, 128)
    runs = []
    for c in cases:
        b = buffers(c)
        ctx = c.create(b[0], stream=side.cuda_stream)
        plan = cb.calvo_window_prepare(ctx, c.requests(), FULL)
        runs.append((c, b, ctx, plan, b[0].clone()))
    torch.cuda.synchronize()

    def step(r):
        _, (pool, q, k, v, q_out, out, lse), _, plan, _ = r
        cb.calvo_kv_append(plan, 0, k[0], v[0], q[0], q_out[0], rope)
        cb.calvo_window_attn(plan, 0, q_out[0], None, None, out[0], lse[0])

    want, graphs = [], []
    for r in runs:
        step(r)
        torch.cuda.synchronize()
        want.append([x.clone() for x in (r[1][0], r[1][4], r[1][5], r[1][6])])
    for r in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(r)
        graphs.append(g)
    for turn in range(4):
        for i, r in enumerate(runs):
            r[1][0].copy_(r[4])
            for x in r[1][4:]:
                x.fill_(3.0)
        torch.cuda.synchronize()
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for i, r in enumerate(runs):
            for x, y in zip((r[1][0], r[1][4], r[1][5], r[1][6]), want[i]):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), turn
        step(runs[turn % 2])                               # eager work between the replays
        torch.cuda.synchronize()
    del graphs, g
    for r in runs:
        cb.calvo_window_destroy(r[3])
        cb.calvo_destroy(r[2])


def test_plans_in_turn_and_calls_without_tokens():
    c = Case8([(40, 2), (7, 1)], 8, 2, 128, seed=8)
    want = c.run(FULL)
    pool, q, k, v, _, out, lse = buffers(c)
    ctx = c.create(pool)
    empty = [cb.calvo_window_prepare(ctx, [], FULL), cb.calvo_window_prepare(ctx, [cb.make_window_request(c.tables[0], 40, 0, -1)], FULL)]
    plans = [cb.calvo_window_prepare(ctx, c.requests(), FULL) for _ in range(3)]
    for p in empty:
        cb.calvo_kv_append(p, 0, None, None)
        cb.calvo_window_attn(p, 0, None, None, None, None, None)
        cb.calvo_window_destroy(p)
    for p in plans:
        cb.calvo_window_attn(p, 0, q[0], k[0], v[0], out[0], lse[0])
    for p in plans:
        cb.calvo_window_destroy(p)
    cb.calvo_destroy(ctx)
    assert torch.equal(out.cpu(), want["out"]) and np.array_equal(pool.cpu().numpy(), want["pool"])


@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_a_pool_of_more_than_4_gib(kind):
    """Blocks at both ends of a pool whose offsets pass 32 bits."""
    c = (Case8 if kind == "e4m3" else Case)([(70, 3), (33, 40)], 32, 8, 128, seed=9)
    nbytes = cb.calvo_block_bytes(8, 128, cb.CALVO_E4M3 if kind == "e4m3" else cb.CALVO_BF16)
    slots = (9 << 29) // nbytes
    move = np.concatenate([np.arange(3), slots - 1 - np.arange(c.slots - 3)]).astype(np.int64)
    f = inv_freq(128)
    small, q, k, v, q_out, out, lse = buffers(c)
    rope = cb.make_rope(torch.from_numpy(f).to(DEV), 128)
    got = []
    for big in (False, True):
        if big:
            pool = torch.zeros((slots, nbytes), dtype=torch.uint8, device=DEV)
            pool[torch.from_numpy(move).to(DEV)] = first
            tables = [move[t].astype(np.int32) for t in c.tables]
        else:
            pool, tables = small.view(torch.uint8).reshape(c.slots, -1), c.tables
            first = pool.clone()
        torch.cuda.synchronize()
        ctx = cb.calvo_create(1, 32, 8, 128, cb.CALVO_E4M3 if kind == "e4m3" else cb.CALVO_BF16, slots if big else c.slots, pool)
        plan = cb.calvo_window_prepare(ctx, [cb.make_window_request(t, a, n, -1) for (a, n), t in zip(c.lens, tables)], FULL)
        cb.calvo_kv_append(plan, 0, k[0], v[0], q[0], q_out[0], rope)
        cb.calvo_window_attn(plan, 0, q_out[0], None, None, out[0], lse[0])
        cb.calvo_window_destroy(plan)
        cb.calvo_destroy(ctx)
        got.append((out.clone(), lse.clone(), pool[torch.from_numpy(move).to(DEV)].clone() if big else pool.clone()))
        del pool
    assert all(torch.equal(x, y) for x, y in zip(*got))


# ---- refusals

def refused(f, code=cb.CALVO_EINVAL, match=None):
    with pytest.raises(cb.CalvoError, match=match) as e:
        f()
    assert e.value.code == code


def test_refusals_of_the_append():
    c = Case8([(20, 3)], 8, 2, 64, seed=10, layers=2)
    pool, q, k, v, q_out, out, lse = buffers(c)
    before, f = pool.clone(), torch.from_numpy(inv_freq(64)).to(DEV)
    rope = lambda *a, **kw: cb.make_rope(*a, **kw)  # noqa: E731
    ctx = c.create(pool)
    plan = cb.calvo_window_prepare(ctx, c.requests(), FULL)
    app = lambda *a: cb.calvo_kv_append(plan, *a)  # noqa: E731
    k0, v0, q0, o0 = k[0], v[0], q[0], q_out[0]
    refused(lambda: app(2, k0, v0), match="layer")
    refused(lambda: app(-1, k0, v0), match="layer")
    refused(lambda: app(0, k0, None), match="both")
    refused(lambda: app(0, None, v0), match="both")
    refused(lambda: app(0, k0, v0, q0), match="both")
    refused(lambda: app(0, k0, v0, None, o0), match="both")
    refused(lambda: app(0, k0.data_ptr() + 2, v0), match="aligned")
    refused(lambda: app(0, k0, v0, q0, o0.data_ptr() + 8), match="aligned")
    for bad in (127, 64, -128, 132, (1 << 41)):
        refused(lambda: app(0, k0, v0, None, None, None, bad), match="stride of k_new")
        refused(lambda: app(0, k0, v0, None, None, None, 0, bad), match="stride of v_new")
    refused(lambda: app(0, None, None, q0, o0, None, 0, 0, 504), match="stride of q")
    refused(lambda: app(0, k0, v0, q0, q0), match="overlap")
    refused(lambda: app(0, k0, v0, q0, k0), match="overlap")
    refused(lambda: app(0, k0, v0, q0, pool.data_ptr()), match="overlap")
    refused(lambda: app(0, pool.data_ptr() + 4096, v0), match="overlap")
    refused(lambda: app(0, k0, v0, q0, o0, rope(q_out, 64)), match="overlap")
    refused(lambda: app(0, k0, v0, q0, o0, rope(f, 64, positions=q_out)), match="overlap")
    for rot in (0, -2, 63, 66, 1):
        refused(lambda: app(0, k0, v0, q0, o0, rope(f, rot)), match="rot_dim")
    refused(lambda: app(0, k0, v0, q0, o0, rope(f, 64, 2)), match="interleaved")
    refused(lambda: app(0, k0, v0, q0, o0, rope(None, 64)), match="inv_freq")
    refused(lambda: app(0, k0, v0, q0, o0, rope(f.data_ptr() + 2, 64)), match="aligned")
    r = rope(f, 64)
    r.reserved = 1
    refused(lambda: app(0, k0, v0, q0, o0, r), match="reserved")
    refused(lambda: cb.calvo_kv_append(None, 0, k0, v0), match="NULL")
    torch.cuda.synchronize()
    assert torch.equal(pool, before) and not q_out.any()
    app(0, k0, v0, q0, o0, rope(f, 64))
    cb.calvo_window_destroy(plan)
    cb.calvo_destroy(ctx)
    assert not torch.equal(pool, before)


def test_what_does_not_take_an_8_bit_pool():
    c = Case8([(32, 3)], 8, 2, 64, seed=10)
    pool, q, k, v, _, out, lse = buffers(c)
    before = pool.clone()
    ctx = c.create(pool, staging_bytes=1 << 20)
    host = torch.zeros(1 << 16, dtype=torch.uint8)
    reqs = [cb.make_request(host, 1 << 16, c.tables[0], 2, 3)]
    cu = np.array([0, 3], np.int32)
    refused(lambda: cb.calvo_prefill_attn(ctx, 0, q[0], k[0], v[0], out[0], reqs, cu), match="8-bit")
    refused(lambda: cb.calvo_prefill_attn_noalloc(ctx, 0, q[0], k[0], v[0], out[0], reqs, cu), match="8-bit")
    refused(lambda: cb.calvo_batch_prepare(ctx, reqs, cu), match="8-bit")
    plan = cb.calvo_window_prepare(ctx, [cb.make_window_request(c.tables[0], 32, 3, 0)], FULL)
    mass = torch.zeros((1, 2, 64), device=DEV)
    refused(lambda: cb.calvo_attn_mass(plan, 0, q[0], lse[0], None, mass, 1, 64), match="8-bit")
    cb.calvo_window_destroy(plan)
    kept = torch.zeros((1, 1, 2, 16), dtype=torch.int32, device=DEV)
    refused(lambda: cb.calvo_kv_evict(ctx, [cb.make_evict_request(c.tables[0], 35, [7], 16)], 0, 1, mass, 1, 64, kept, 16), match="8-bit")
    from paper_2603_21257_amd import dispatch
    with pytest.raises(cb.CalvoError, match="8-bit"):
        dispatch.Dispatcher(ctx, cb.CALVO_POLICY_SJF, (1e-6, 0.0, 1e-6, 0.0))
    cb.calvo_destroy(ctx)
    assert torch.equal(pool, before) and not out.any()
    with pytest.raises(cb.CalvoError, match="multiple of 16"):
        cb.calvo_create(1, 8, 2, 40, cb.CALVO_E4M3, 4, pool)
