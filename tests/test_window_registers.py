"""The compiled window kernels: the pipelined ones keep the wait states around their MFMAs (test_attn_registers.py) and spill nothing, none has
scratch memory (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2603_21257_amd import build as b
from test_attn_registers import Code, compiled


@pytest.mark.parametrize("kernel,mfmas,exps,turns", [("window_pipe_kernel", 64, 32, 8), ("window_duo_kernel", 32, 16, 10)])
def test_pipelined(kernel, mfmas, exps, turns, tmp_path):
    usage, asm = compiled("attn_window_pipe.hip", kernel, tmp_path)
    assert re.search(r"VGPRs Spill: 0\b", usage) and re.search(r"ScratchSize \[bytes/lane\]: 0\b", usage), usage
    steady = [x for x in re.split(r"^\.LBB\w+:", asm, flags=re.M) if x.count("v_mfma") == mfmas and x.count("v_exp_f32") == exps]
    assert len(steady) >= turns
    assert all("v_accvgpr" not in x for x in steady)
    code = Code(asm, kernel)
    assert sum(x.mfma for x in code.ins) >= turns * mfmas
    assert code.hazards() == []


@pytest.mark.parametrize("source", ["attn_window.hip", "attn_mass.hip", "kv_evict.hip"])
def test_no_scratch_memory(source, tmp_path):
    flags = [f for f in b.FLAGS if f != "-shared"]
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "--cuda-device-only", "-S", os.path.join(b.CSRC, source), "-o",
                        str(tmp_path / "k.s")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    asm = (tmp_path / "k.s").read_text()
    sizes = re.findall(r"\.private_segment_fixed_size: (\d+)\n", asm)
    assert sizes and set(sizes) == {"0"}
