"""Buffer loads that rely on the bounds of their resource (no GPU needed): the hardware compares the vector offset and the immediate with the number of
bytes, the scalar offset is not part of the comparison.  None of the compiled kernels has one."""
import os
import re
import subprocess

import pytest

from paper_2603_21257_amd import build as b


@pytest.mark.parametrize("source", ["kv_evict.hip", "attn_mass.hip", "attn_window.hip", "attn_rows.hip"])
def test_no_scalar_offsets(source, tmp_path):
    flags = [f for f in b.FLAGS if f != "-shared"]
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--cuda-device-only", "-S", os.path.join(b.CSRC, source), "-o",
                        str(tmp_path / "k.s")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    loads = re.findall(r"^\s*(buffer_(?:load|store)\S* .*)$", (tmp_path / "k.s").read_text(), re.M)
    assert loads
    # data, vector offset, resource, scalar offset [offen] [offset:n]
    scalar = [x for x in loads if not re.match(r"\S+\s+\S+, \S+, s\[\d+:\d+\], 0( |$)", x)]
    assert not scalar, f"{len(scalar)} of {len(loads)}, first: {scalar[0]}"
