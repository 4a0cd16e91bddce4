"""The waves of a workgroup that appends to an 8-bit pool meet at the same barrier, whatever each of them stores (no GPU needed)."""
import os
import re
import subprocess

from paper_2603_21257_amd import build as b


def test_one_barrier_for_k_and_v(tmp_path):
    """Rows of q: one barrier, and one behind the angles; blocks: one."""
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *[f for f in b.FLAGS if f != "-shared"], "--cuda-device-only", "-S",
                        os.path.join(b.CSRC, "kv_append.hip"), "-o", str(tmp_path / "k.s")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    asm = (tmp_path / "k.s").read_text()
    found = re.findall(r"^(\w*append_e4m3_kernelILi(\d+)ELi(\d+)E\w*):(.*?)^\.Lfunc_end", asm, flags=re.M | re.S)
    assert len(found) >= 14                              # three widths, the orders of pairs
    for _, dim, mode, code in found:
        assert len(re.findall(r"\ts_barrier\b", code)) == (2 if mode == "0" else 3), (dim, mode)
