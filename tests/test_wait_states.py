"""The compiled block operators hold no result read too early and no copy under a partial mask."""
import os
import subprocess

import pytest
import wait_states as W

from paper_2502_19864_amd import build


def _one(text):
    (_, ins, labels), = W.kernels("_Zk:\n" + text)
    return ins, labels


def test_a_short_way_behind_two_branches_is_found():
    text = """
	v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], 0
	s_cbranch_vccnz .LBB0_2
	s_nop 6
	s_branch .LBB0_3
.LBB0_2:
	v_mov_b32_e32 v9, v8
.LBB0_3:
	s_nop %d
	v_accvgpr_read_b32 v10, a15
	s_endpgm
"""
    assert [x[2] for x in W.short_waits(*_one(text % 3))] == [6]
    assert not W.short_waits(*_one(text % 8))


def test_a_copy_ahead_of_the_mask_is_found():
    text = """
	s_and_saveexec_b64 s[0:1], vcc
	s_cbranch_execz .LBB0_2
	v_add_u32_e32 v1, v1, v2
.LBB0_2:
	%s
	s_or_b64 exec, exec, s[0:1]
	s_endpgm
"""
    assert len(W.masked_copies(*_one(text % "v_accvgpr_write_b32 a9, v11"))) == 1
    assert not W.masked_copies(*_one(text % "s_nop 0"))


@pytest.mark.parametrize("source", ["k_attn_masked.hip"])
def test_compiled_kernels(source, tmp_path):
    out = str(tmp_path / "k.s")
    subprocess.run([build.hipcc()] + build.flags() + ["-S", "--cuda-device-only", os.path.join(build.CSRC, source),
                                                     "-o", out], check=True, capture_output=True)
    n = 0
    for name, ins, labels in W.kernels(open(out).read()):
        n += 1
        assert not W.short_waits(ins, labels), name
        assert not W.masked_copies(ins, labels), name
    assert n > 60
