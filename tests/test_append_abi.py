"""calvo_rope as a C compiler lays it out, and calls that hold before any device work (no GPU needed)."""
import ctypes
import os
import subprocess

import pytest

from paper_2603_21257_amd import binding as cb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rope_layout(tmp_path):
    st = cb.calvo_rope
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "calvo.h"', 'int main(void) {', '  printf("size %zu\\n", sizeof(calvo_rope));']
    lines += [f'  printf("{n} %zu\\n", offsetof(calvo_rope, {n}));' for n, _ in st._fields_]
    (tmp_path / "l.c").write_text("\n".join(lines + ['  return 0;', '}']))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = dict(ln.split() for ln in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(out["size"]) == ctypes.sizeof(st)
    for n, _ in st._fields_:
        assert int(out[n]) == getattr(st, n).offset


def test_null_arguments():
    with pytest.raises(cb.CalvoError) as e:
        cb.calvo_kv_append(0, 0, None, None)
    assert e.value.code == cb.CALVO_EINVAL and "window is NULL" in str(e.value)
    assert cb.lib().calvo_block_bytes(None, None) == cb.CALVO_EINVAL
