"""Window batches and evictions on the host (no GPU needed): every key that a row sees is met once, what the kernels take for visible to all rows is,
and bad requests are refused."""
import os
import subprocess

import numpy as np
import pytest

from paper_2603_21257_amd import binding as cb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FULL = (1 << 31) - 1
B = 16


def tables(lens, seed=0):
    perm = np.random.default_rng(seed).permutation(sum(-(-n // B) for n in lens) + 3).astype(np.int32)
    at = np.cumsum([0] + [-(-n // B) for n in lens])
    return [perm[a:b] for a, b in zip(at[:-1], at[1:])], len(perm)


def plan(lens, window, n_first, hq=8, hkv=2, dim=128, dtype=cb.CALVO_BF16, n_cus=256):
    tabs, slots = tables([c + n for c, n in lens])
    reqs = [cb.make_window_request(t, c, n, i) for i, (t, (c, n)) in enumerate(zip(tabs, lens))]
    return cb.calvo_window_plan(hq, hkv, dim, dtype, max(slots, 1), n_cus, reqs, window, n_first)


def check(lens, window, n_first, hq=8, hkv=2, dim=128, dtype=cb.CALVO_BF16, n_cus=256):
    _, e = plan(lens, window, n_first, hq, hkv, dim, dtype, n_cus)
    g = hq // hkv
    for r, (c, n) in enumerate(lens):
        mine = e[e[:, 0] == r]
        rows = np.arange(n * g)
        met = np.zeros((n * g, -(-(c + n) // 32) + 1), np.int32)
        for _, a, b, s0, s1, full, _ in mine:
            assert 0 <= a < b <= n * g and 0 <= s0 < s1 <= met.shape[1] - 1
            met[a:b, s0:s1] += 1
            if full:
                pos = c + np.array([a, b - 1]) // g
                t = np.arange(32 * s0, 32 * s1)
                assert (t <= pos[0]).all() and ((t > pos[1] - window) | (t < n_first)).all()
        assert met.max(initial=0) <= 1, "a sub-tile twice"
        t = np.arange(c + n)
        pos = (c + rows // g)[:, None]
        sees = (t[None] <= pos) & ((t[None] > pos - window) | (t[None] < n_first))
        need = np.zeros_like(met, dtype=bool)
        i, k = np.nonzero(sees)
        need[i, k // 32] = True
        assert (met[need] == 1).all(), "a visible key is not met"


@pytest.mark.parametrize("shape", [(8, 2, 128, cb.CALVO_BF16), (5, 1, 128, cb.CALVO_BF16), (8, 8, 64, cb.CALVO_BF16), (6, 3, 256, cb.CALVO_F32)])
@pytest.mark.parametrize("variant", ["", "3", "4", "5"])
def test_visible_keys_are_met_once(shape, variant, monkeypatch):
    monkeypatch.setenv("CALVO_ATTN_VARIANT", variant)
    hq, hkv, dim, dtype = shape
    rng = np.random.default_rng(3)
    for window, n_first in [(1, 0), (5, 3), (31, 32), (64, 4), (100, 200), (300, 17), (FULL, 0), (40, FULL), (1000, 31)]:
        for lens in [[(0, 1)], [(0, 70)], [(1000, 1)], [(1003, 130), (0, 0), (17, 0), (31, 2)], [(int(rng.integers(0, 3000)), int(rng.integers(1, 300)))]]:
            for n_cus in (1, 256):
                check(lens, window, n_first, hq, hkv, dim, dtype, n_cus)


def test_a_short_window_is_little_work():
    """Sub-tiles of a token behind a window do not grow with its context."""
    for c in (5000, 50000, 300000):
        _, e = plan([(c, 1)], 1024, 4, n_cus=1)
        assert int((e[:, 4] - e[:, 3]).sum()) <= 1024 // 32 + 3


def test_tokens_behind_the_32_bit_range_of_bytes():
    _, e = plan([(1 << 20, 3)], 100, 5)
    assert e[:, 4].max() == ((1 << 20) + 3 + 31) // 32


def refused(code, text, f):
    with pytest.raises(cb.CalvoError) as err:
        f()
    assert err.value.code == code and text in str(err.value), err.value


def request(c=20, n=2, table=None, row=0, reserved=0):
    r = cb.make_window_request(np.arange(8) if table is None else table, c, n, row)
    r.reserved = reserved
    return r


def window_plan(reqs, window=10, n_first=0, blocks=8, dim=64):
    return cb.calvo_window_plan(8, 2, dim, cb.CALVO_BF16, blocks, 256, reqs, window, n_first)


def test_window_refusals():
    window_plan([request()])
    window_plan([])
    refused(cb.CALVO_EINVAL, "window", lambda: window_plan([request()], window=0))
    refused(cb.CALVO_EINVAL, "n_first", lambda: window_plan([request()], n_first=-1))
    refused(cb.CALVO_EINVAL, "negative", lambda: window_plan([request(-1, 2)]))
    refused(cb.CALVO_EINVAL, "negative", lambda: window_plan([request(3, -2)]))
    refused(cb.CALVO_EINVAL, "outside the pool", lambda: window_plan([request(20, 2, [0, 8])]))
    refused(cb.CALVO_EINVAL, "outside the pool", lambda: window_plan([request(20, 2, [0, -1])]))
    refused(cb.CALVO_EINVAL, "twice", lambda: window_plan([request(20, 2, [3, 3])]))
    refused(cb.CALVO_ENOMEM, "slots", lambda: window_plan([request(120, 9, np.arange(9))]))
    refused(cb.CALVO_EINVAL, "reserved", lambda: window_plan([request(reserved=1)]))
    r = request()
    r.block_table = None
    refused(cb.CALVO_EINVAL, "NULL", lambda: window_plan([r]))
    r = request()
    r.n_cached = (1 << 31) - 100
    refused(cb.CALVO_EINVAL, "too long", lambda: window_plan([r]))
    refused(cb.CALVO_EINVAL, "head_dim", lambda: window_plan([request()], dim=68))
    with pytest.raises(ValueError):
        cb.make_window_request([0], 16, 1)


def test_slots_that_take_new_tokens_are_in_one_table():
    shared = [0, 1, 2]
    window_plan([request(48, 2, shared + [3]), request(48, 2, shared + [4])])           # a run of whole blocks that is only read
    window_plan([request(20, 0, [5, 6]), request(40, 0, [5, 6, 7])])                    # nobody stores
    refused(cb.CALVO_EINVAL, "new tokens", lambda: window_plan([request(40, 2, shared), request(40, 2, shared)]))
    refused(cb.CALVO_EINVAL, "new tokens", lambda: window_plan([request(40, 2, shared), request(40, 0, shared)]))
    refused(cb.CALVO_EINVAL, "new tokens", lambda: window_plan([request(40, 0, shared), request(40, 2, shared)]))
    refused(cb.CALVO_EINVAL, "new tokens", lambda: window_plan([request(32, 2, shared), request(48, 3, [2, 4, 5, 6])]))


def evict(n=40, keep=20, first=1, last=2, src=(0, 1, 2), dst=(3, 4), row=0, reserved=0):
    r = cb.make_evict_request(list(src), n, list(dst), keep, first, last, row)
    r.reserved = reserved
    return r


def evict_check(*reqs, rows=2, blocks=8):
    cb.calvo_evict_check(2, 64, cb.CALVO_F32, blocks, list(reqs), rows)


def test_evict_refusals():
    evict_check()
    evict_check(evict())
    evict_check(evict(keep=0, first=0, last=0, dst=()), evict())
    evict_check(evict(), evict(dst=(5, 6), row=1))                                       # one source, two destinations
    refused(cb.CALVO_EINVAL, "keeps", lambda: evict_check(evict(n=10, keep=11)))
    refused(cb.CALVO_EINVAL, "negative", lambda: evict_check(evict(first=-1)))
    refused(cb.CALVO_EINVAL, "n_first + n_last", lambda: evict_check(evict(first=10, last=11)))
    refused(cb.CALVO_EINVAL, "outside the pool", lambda: evict_check(evict(src=(0, 1, 8))))
    refused(cb.CALVO_EINVAL, "outside the pool", lambda: evict_check(evict(dst=(3, -1))))
    refused(cb.CALVO_EINVAL, "twice", lambda: evict_check(evict(src=(0, 1, 1))))
    refused(cb.CALVO_EINVAL, "twice", lambda: evict_check(evict(dst=(4, 4))))
    refused(cb.CALVO_EINVAL, "twice", lambda: evict_check(evict(), evict(dst=(4, 5), row=1)))
    refused(cb.CALVO_EINVAL, "in a dst_table", lambda: evict_check(evict(dst=(2, 4))))
    refused(cb.CALVO_EINVAL, "in a dst_table", lambda: evict_check(evict(), evict(src=(3, 5, 6), dst=(7, 1), row=1)))
    refused(cb.CALVO_EINVAL, "mass_row", lambda: evict_check(evict(row=2)))
    refused(cb.CALVO_EINVAL, "differ", lambda: evict_check(evict(), evict(dst=(5, 6))))
    refused(cb.CALVO_EINVAL, "reserved", lambda: evict_check(evict(reserved=3)))
    refused(cb.CALVO_ENOMEM, "slots", lambda: evict_check(evict(), blocks=4))
    with pytest.raises(ValueError):
        cb.make_evict_request([0], 16, [], 1)


@pytest.mark.parametrize("name,args", [("calvo_window_prepare", (None, None, 0, 1, 0, None)), ("calvo_window_destroy", (None,)),
                                       ("calvo_window_attn", (None, 0, None, None, None, None, None, 0.0)),
                                       ("calvo_attn_mass", (None, 0, None, None, None, None, 0, 0, 0, 0.0)),
                                       ("calvo_kv_evict", (None, None, 0, 0, 0, None, 0, 0, None, 0, None, 0)),
                                       ("calvo_window_plan", (None, 1, None, 0, 1, 0, None, None, 0, None)), ("calvo_evict_check", (None, None, 0, 0))])
def test_null_handles(name, args):
    assert getattr(cb.lib(), name)(*args) == cb.CALVO_EINVAL


def test_struct_layouts(tmp_path):
    structs = [cb.calvo_window_request, cb.calvo_evict_request]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "calvo.h"', 'int main(void) {']
    for st in structs:
        lines.append(f'  printf("{st.__name__} %zu\\n", sizeof({st.__name__}));')
        lines += [f'  printf("{st.__name__}.{n} %zu\\n", offsetof({st.__name__}, {n}));' for n, _ in st._fields_]
    (tmp_path / "l.c").write_text("\n".join(lines + ['  return 0;', '}']))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = dict(ln.split() for ln in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines())
    import ctypes
    for st in structs:
        assert int(out[st.__name__]) == ctypes.sizeof(st)
        for n, _ in st._fields_:
            assert int(out[f"{st.__name__}.{n}"]) == getattr(st, n).offset
