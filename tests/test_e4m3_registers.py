"""The compiled kernels over 8-bit pools: the pipelined ones keep the wait states around their MFMAs (test_attn_registers.py) and spill nothing, none has
scratch memory (no GPU needed)."""
import re

import pytest

from test_attn_registers import Code, compiled
import test_window_registers


# turns: steps of the unrolled loop, as many as the ring has slots (8 and 4; an odd ring's would be unrolled twice)
@pytest.mark.parametrize("kernel,mfmas,exps,turns", [("e4m3_pipe_kernel", 64, 32, 8), ("e4m3_duo_kernel", 32, 16, 4)])
def test_pipelined(kernel, mfmas, exps, turns, tmp_path):
    usage, asm = compiled("attn_e4m3_pipe.hip", kernel, tmp_path)
    assert re.search(r"VGPRs Spill: 0\b", usage) and re.search(r"ScratchSize \[bytes/lane\]: 0\b", usage), usage
    steady = [x for x in re.split(r"^\.LBB\w+:", asm, flags=re.M) if x.count("v_mfma") == mfmas and x.count("v_exp_f32") == exps]
    assert len(steady) >= turns
    assert all("v_accvgpr" not in x and x.count("v_cvt_scalef32") == 16 for x in steady)
    code = Code(asm, kernel)
    assert sum(x.mfma for x in code.ins) >= turns * mfmas
    assert code.hazards() == []


@pytest.mark.parametrize("source", ["attn_e4m3.hip", "kv_append.hip"])
def test_kernels_without_scratch_memory(source, tmp_path):
    test_window_registers.test_no_scratch_memory(source, tmp_path)
