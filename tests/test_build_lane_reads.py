"""The check of the build's assembly: what has to wait before a lane of another's register is read, on small listings of both kinds."""
import pytest

from paper_2104_14129_amd import build

READ = "v_fmac_f32_dpp v1, v2, v3 row_newbcast:4 row_mask:0xf bank_mask:0xf"


@pytest.mark.parametrize("before", [
    ["v_mov_b32_e32 v2, v9", "s_nop 1"],
    ["v_add_f32_e32 v2, v9, v8", "v_mov_b32_e32 v7, v6", "s_mov_b32 s0, s1"],
    ["ds_read_b128 v[0:3], v9", "s_waitcnt lgkmcnt(0)"],                          # the compiler's wait counts hold for operands
    ["v_exp_f32_e32 v3, v9", "s_nop 0"],
    ["v_exp_f32_e32 v9, v8"],
    ["v_mov_b32_e32 v1, 0", "v_mov_b32_e32 v3, 0"],                               # not read from another lane
    ["v_mfma_f32_16x16x32_f16 v[0:3], v[8:11], v[12:15], 0", "s_nop 7", "s_nop 7", "s_nop 1"],
    ["v_mfma_f32_16x16x32_f16 v[0:3], v[8:11], v[12:15], 0", "v_mul_f32_dpp v1, v9, v1 row_newbcast:4", "v_mov_b32_e32 v4, v3", "v_mul_f32_e32 v3, v3, v4", "v_mul_f32_e32 v2, v2, v4", "s_nop 1"],
    ["v_mov_b32_e32 v[20:23], v9"],
    [".LBB0_1:", "s_nop 1"],
])
def test_what_waits_long_enough(before):
    assert build.lane_read_hazards("\n".join("\t" + t for t in ["s_nop 7"] * 3 + before + [READ])) == []


@pytest.mark.parametrize("before", [
    ["v_mov_b32_e32 v2, v9"],
    ["v_mov_b32_e32 v2, v9", "s_nop 0"],
    ["v_add_f32_e32 v2, v9, v8", "v_mov_b32_e32 v7, v6"],
    ["s_nop 1", "v_mov_b32_e32 v2, v9"],                                          # a copy behind the wait
    ["v_accvgpr_read_b32 v2, a0"],
    ["v_pk_mov_b32 v[2:3], v[4:5], v[6:7]", "s_nop 0"],
    ["v_exp_f32_e32 v3, v9"],
    ["v_rcp_f32_e32 v1, v9"],
    ["v_mfma_f32_16x16x32_f16 v[0:3], v[8:11], v[12:15], 0", "s_nop 7"],
    ["v_cmpx_gt_f32_e32 v8, v9", "s_nop 3"],
    [".LBB0_1:", "s_mov_b32 s0, s1"],
    [".LBB0_1:"],
])
def test_what_does_not(before):
    assert len(build.lane_read_hazards("\n".join("\t" + t for t in ["s_nop 7"] * 3 + before + [READ]))) >= 1
