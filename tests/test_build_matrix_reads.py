"""The build looks through the device listings for results of matrix instructions that are read before they are there.  Small listings, written by
hand.  No GPU."""
import pytest

from paper_2603_09221_amd import build

BODY = """
a_kernel:                               ; @a_kernel
; %%bb.0:
	v_mfma_f32_16x16x4_f32 a[8:11], v12, v7, a[8:11]
	s_cbranch_vccnz .LBB0_2
; %%bb.1:
	v_mfma_f32_16x16x4_f32 a[0:3], v12, v7, a[0:3]
	s_nop 9
.LBB0_2:                                ;   in Loop: Header
	%s
	ds_read_b128 v[4:7], v32
	%s
	s_nop 6
	v_accvgpr_read_b32 v220, a10
	s_endpgm
"""
NOTHING = "s_waitcnt lgkmcnt(0)"


@pytest.mark.parametrize("read", ["v_accvgpr_read_b32 v221, a11", "v_add_f32_e32 v1, v2, a8", "ds_write_b128 v3, a[8:11]", "global_store_dword v[2:3], a9, off"])
def test_a_read_behind_a_skipped_block_is_found(read):
    """The branch is one wait state, the read of LDS another: eight are needed."""
    for text in (BODY % (read, NOTHING), BODY % (NOTHING, read)):
        assert [(k, x) for k, _, x in build.early_matrix_reads(text)] == [("a_kernel", read)]
    assert not build.early_matrix_reads(BODY % ("s_nop 7", read))
    assert not build.early_matrix_reads(BODY % (NOTHING, NOTHING))


def test_other_registers_and_further_products_are_left_alone():
    for line in ("v_accvgpr_read_b32 v221, a12", "v_accvgpr_write_b32 a20, v8", "v_mov_b32_e32 v8, v9"):
        assert not build.early_matrix_reads(BODY % (NOTHING, line)), line
    again = BODY % ("v_mfma_f32_16x16x4_f32 a[8:11], v12, v7, a[8:11]", "v_accvgpr_read_b32 v221, a11")
    assert [n for _, n, _ in build.early_matrix_reads(again)] == [12]     # of the second product alone
    overwritten = BODY % ("v_accvgpr_write_b32 a11, v8", "v_accvgpr_read_b32 v221, a11")
    assert not build.early_matrix_reads(overwritten)


def test_shapes_differ_in_what_they_take():
    text = "a_kernel:\n\tv_mfma_f32_%s v[0:3], v12, v7, v[0:3]\n\ts_nop %d\n\tv_add_f32_e32 v9, v9, v3\n\ts_endpgm\n"
    for shape, passes in (("16x16x32_bf16", 4), ("32x32x16_bf16", 8), ("16x16x4_f32", 8), ("32x32x2_f32", 16)):
        assert build.early_matrix_reads(text % (shape, passes - 2)) and not build.early_matrix_reads(text % (shape, passes - 1))
