"""asm_check.py on the scaled matrix instruction, whose exponents are vector registers like its operands (no GPU needed)."""
import os

import pytest

from paper_2502_02581_amd import asm_check, build

MFMA = "v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[2:9], v[10:17], a[0:3], v18, v19 op_sel_hi:[0,0,0]"


@pytest.mark.parametrize("writer,found", [("v_and_b32_e32 v19, 0xff, v20", True), ("v_mov_b32_e32 v18, v1", True), ("v_mov_b32_e32 v5, v1", True),
                                          ("v_mov_b32_e32 v12, v1", True), ("v_mov_b32_e32 v20, v1", False), ("ds_read_b32 v19, v1", False)])
def test_writers_right_before_the_instruction(writer, found):
    assert bool(asm_check.check_mfma_sources([writer, MFMA])) == found
    assert not asm_check.check_mfma_sources([writer, "s_nop 1", MFMA])


def test_current_build_passes():
    path = build.device_asm("quant_expert.hip")
    if not os.path.exists(path):
        pytest.skip("the assembly of the last build is not here")
    text = open(path).read()
    assert text.count("v_mfma_scale_f32_16x16x128_f8f6f4") > 1000
    assert asm_check.check(path) == []
