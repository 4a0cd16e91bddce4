"""The buffers of plans and evictions that were given back (csrc/step_bufs.h), over a made-up device that is some steps behind (no GPU needed)."""
import os
import subprocess

import pytest

from paper_2603_21257_amd import build as b

SOURCE = r"""
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <set>
#include "step_bufs.h"

#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

struct Buf { size_t d_bytes = 0, h_bytes = 0; long read = -1; bool pending = false; int id = 0; };

struct Dev {
  long now = 0, behind = 2, makes = 0, frees = 0, waits = 0, fail = 0;
  size_t held = 0, most = 0;
  std::set<int> alive;
  int make(Buf& b) {
    if (fail > 0) { fail--; return 7; }
    b.id = (int)++makes;
    alive.insert(b.id);
    held += b.d_bytes + b.h_bytes;
    most = std::max(most, held);
    return 0;
  }
  void free(Buf& b) {
    if (b.id) { CHECK(alive.erase(b.id) == 1); held -= b.d_bytes + b.h_bytes; frees++; }
    b = Buf();
  }
  bool was_read(Buf& b) { return b.read <= now - behind; }
  int wait(Buf& b) { waits++; return b.read <= now ? 0 : 9; }
};

// one plan: taken, read by the device, given back
void use(calvo::StepBufs<Buf>& l, Dev& dev, size_t d, size_t h) {
  Buf x;
  CHECK(l.take(dev, d, h, x) == 0 && x.id && !x.pending && x.d_bytes >= d && x.h_bytes >= h);
  x.read = dev.now;
  x.pending = true;
  const long frees = dev.frees, waits = dev.waits;
  CHECK(l.give(x) && !x.id);
  CHECK(dev.frees == frees && dev.waits == waits);
}

// words of a decoding step's descriptors and tables
size_t words_of(int reqs, double lo, double hi, long step) {
  size_t words = 0;
  for (int r = 0; r < reqs; r++) {
    const long n = (long)(lo * std::pow(hi / lo, reqs > 1 ? (double)r / (reqs - 1) : 0)) + step;
    words += n / 16 + 2 + (n / 256 + 1) * 12 + 16;
  }
  return words;
}

int main() {
  {
    // contexts that grow: a few buffers per doubling, and no wait on the host
    struct { int reqs; double lo, hi; } runs[] = {{1, 16, 16}, {64, 2000, 2000}, {128, 300, 33000}, {256, 300, 33000}};
    for (auto& x : runs) {
      for (long behind : {0, 2, 3}) {
        calvo::StepBufs<Buf> l;
        Dev dev;
        dev.behind = behind;
        for (dev.now = 0; dev.now < 16000; dev.now++) {
          const size_t bytes = words_of(x.reqs, x.lo, x.hi, dev.now) * 4;
          use(l, dev, bytes, bytes);
        }
        printf("%d requests, %ld behind: %ld made, %ld freed, %ld waits\n", x.reqs, behind, dev.makes, dev.frees, dev.waits);
        CHECK(dev.makes <= 40 && dev.frees <= 40 && dev.waits == 0);
        l.clear(dev);
        CHECK(dev.alive.empty() && dev.held == 0);
      }
    }
  }
  {
    // many plans at once, then larger ones: what is too small for them goes, and each is found again
    calvo::StepBufs<Buf> l;
    Dev dev;
    std::vector<Buf> many(70);
    for (Buf& x : many) CHECK(l.take(dev, 100, 100, x) == 0);
    CHECK(dev.makes == 70);
    for (Buf& x : many) CHECK(l.give(x));
    CHECK(dev.frees == 0);
    for (int i = 0; i < 100; i++, dev.now++) use(l, dev, 3 << 20, 2 << 20);
    CHECK(dev.makes <= 74 && (long)dev.alive.size() <= 16 + 4);
    const long makes = dev.makes;
    for (int i = 0; i < 100; i++, dev.now++) {
      use(l, dev, 100, 100);
      use(l, dev, 3 << 20, 2 << 20);
    }
    CHECK(dev.makes <= makes + 4);
    l.clear(dev);
    CHECK(dev.alive.empty());
  }
  {
    // large partial results: what is kept beside a new buffer is bounded
    calvo::StepBufs<Buf> l;
    Dev dev;
    for (size_t mb = 1; mb <= 400; mb += 3, dev.now++) use(l, dev, mb << 20, 4096);
    CHECK(dev.held <= ((size_t)256 + 5 * 432) << 20 && dev.makes <= 80);
    l.clear(dev);
    CHECK(dev.held == 0);
  }
  {
    // steps ahead of a device that has read nothing: a few of a size, then the oldest is waited for
    calvo::StepBufs<Buf> l;
    Dev dev;
    dev.behind = 1000;
    for (; dev.now < 50; dev.now++) use(l, dev, 100, 100);
    CHECK(dev.makes == calvo::StepBufs<Buf>::kInTurn && dev.waits == 50 - dev.makes);
    l.clear(dev);
  }
  {
    // no memory: what was given back goes, then the error is the caller's
    calvo::StepBufs<Buf> l;
    Dev dev;
    use(l, dev, 100, 100);
    dev.fail = 1;
    use(l, dev, 1 << 20, 100);
    CHECK(dev.makes == 2 && dev.frees == 1);
    dev.fail = 2;
    Buf x;
    CHECK(l.take(dev, 1 << 24, 100, x) == 7 && !x.id && dev.alive.empty());
  }
  CHECK(calvo::step_buf_size(0, 65536) == 65536 && calvo::step_buf_size(65537, 65536) == 131072 && calvo::step_buf_size((size_t)16 << 20, 65536) == (size_t)16 << 20);
  CHECK(calvo::step_buf_size(((size_t)16 << 20) + 1, 65536) == (size_t)32 << 20 && calvo::step_buf_size(((size_t)5 << 32) + 5, 65536) == ((size_t)5 << 32) + ((size_t)16 << 20));
  return 0;
}
"""


def test_buffers_given_back(tmp_path):
    (tmp_path / "t.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-I", b.CSRC, str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    r = subprocess.run([str(tmp_path / "t")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=100, env={k: v for k, v in os.environ.items() if k != "LD_PRELOAD"})
    print(r.stdout)
    assert r.returncode == 0, r.stdout


@pytest.mark.gpu
def test_a_larger_plan_behind_many_small_ones():
    """70 plans at once, then one with a table of 2 MB again and again: its buffer is there the second time, and is not handed back to the device in between."""
    import numpy as np
    import torch

    from paper_2603_21257_amd import binding as cb
    slots = 1 << 19
    pool = torch.zeros((1, slots, 2, 16, 1, 8), dtype=torch.bfloat16, device="cuda:0")
    table = np.arange(slots, dtype=np.int32)
    torch.cuda.synchronize()
    ctx = cb.calvo_create(1, 1, 1, 8, cb.CALVO_BF16, slots, pool)

    def free():
        torch.cuda.synchronize()
        return torch.cuda.mem_get_info()[0]

    try:
        small = [cb.calvo_window_prepare(ctx, [cb.make_window_request(table[:2], 20, 1, -1)], 10) for _ in range(70)]
        for p in small:
            cb.calvo_window_destroy(p)
        large = [cb.make_window_request(table, 16 * slots - 1, 1, -1)]
        held = []
        for _ in range(3):
            p = cb.calvo_window_prepare(ctx, large, 10)
            held.append(free())
            cb.calvo_window_destroy(p)
            held.append(free())
        assert len(set(held)) == 1, held
    finally:
        cb.calvo_destroy(ctx)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
def test_steps_ahead_of_the_device(dim):
    """Decoding steps of requests whose tables outgrow several sizes of buffers, with chunks and evictions in between: the same bits whether the host waits after each
    call or for none."""
    import numpy as np
    import torch

    from paper_2603_21257_amd import binding as cb
    hq, hkv, steps, blocks = 8, 2, 40, 9000
    slots = 3 * blocks
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(3)
    start = torch.randn((1, slots + 8, 2, 16, hkv, dim), dtype=torch.float32, device="cuda:0", generator=gen).to(torch.bfloat16)
    q = torch.randn((steps, 70, hq, dim), dtype=torch.float32, device="cuda:0", generator=gen).to(torch.bfloat16)
    k, v = (torch.randn((steps, 70, hkv, dim), dtype=torch.float32, device="cuda:0", generator=gen).to(torch.bfloat16) for _ in range(2))
    tables = np.random.default_rng(2).permutation(slots).astype(np.int32).reshape(3, blocks)

    def run(wait):
        pool = start.clone()
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:-1], device="cuda:0")
        stride = 16 * blocks
        mass = torch.zeros((1, 3, hkv, stride), device="cuda:0")
        kept = torch.zeros((steps, 1, hkv, 100), dtype=torch.int32, device="cuda:0")
        torch.cuda.synchronize()
        ctx = cb.calvo_create(1, hq, hkv, dim, cb.CALVO_BF16, slots + 8, pool)
        done = (lambda: torch.cuda.synchronize()) if wait else (lambda: None)
        try:
            for s in range(steps):
                # one request has a chunk in every eighth step, the others a token; contexts grow by a quarter a step
                lens = [(min(16 * blocks - 80, int(40 * 1.25 ** s) + 7 * r), 64 if s % 8 == 5 and r == 1 else 1) for r in range(3)]
                p = cb.calvo_window_prepare(ctx, [cb.make_window_request(t, c, n, r) for r, (t, (c, n)) in enumerate(zip(tables, lens))], 300, 4)
                done()
                cb.calvo_window_attn(p, 0, q[s], k[s], v[s], out[s], lse[s])
                done()
                cb.calvo_attn_mass(p, 0, q[s], lse[s], mass, mass, 3, stride)
                done()
                cb.calvo_window_destroy(p)
                if lens[0][0] > 100:
                    cb.calvo_kv_evict(ctx, [cb.make_evict_request(tables[0], lens[0][0], np.arange(slots, slots + 7), 100, 4, 16)], 0, 1, mass, 3, stride, kept[s], 100)
                    done()
        finally:
            cb.calvo_destroy(ctx)
        torch.cuda.synchronize()
        return [x.view(torch.int16) if x.dtype == torch.bfloat16 else x for x in (out, lse, mass, kept, pool)]

    assert all(torch.equal(a, b) for a, b in zip(run(True), run(False)))
