"""The build scans the device assembly for results of matrix instructions that are touched before they are written.  The scanner against
hand-written fragments."""
from paper_2311_15269_amd.build import early_reads_of_products

PRODUCT = "\tv_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]\n"


def test_a_read_right_behind_is_reported():
    assert early_reads_of_products(PRODUCT + "\tv_accvgpr_read_b32 v9, a15\n") == ["2: v_accvgpr_read_b32 v9, a15"]


def test_other_registers_and_further_products_pass():
    assert early_reads_of_products(PRODUCT + "\tv_accvgpr_read_b32 v9, a16\n\tv_add_f32 v15, v16, v17\n" + PRODUCT) == []


def test_time_passes():
    assert early_reads_of_products(PRODUCT + "\ts_nop 9\n\tv_accvgpr_read_b32 v9, a0\n") != []
    assert early_reads_of_products(PRODUCT + "\ts_nop 10\n\tv_accvgpr_read_b32 v9, a0\n") == []
    assert early_reads_of_products(PRODUCT + "\ts_add_i32 s0, s0, 1\n" * 11 + "\tv_accvgpr_read_b32 v9, a0\n") == []
    assert early_reads_of_products(PRODUCT + "\tv_mfma_f32_32x32x16_bf16 a[16:31], v[0:3], v[4:7], a[16:31]\n" * 2 + "\tv_mov_b32 v9, a0\n") == []


def test_the_way_back_of_a_loop_counts():
    asm = "LBB0_1:\n\tv_accvgpr_read_b32 v9, a15\n" + "\ts_nop 15\n" + PRODUCT + "\ts_add_i32 s0, s0, 1\n\ts_cbranch_scc1 LBB0_1\n\ts_endpgm\n"
    assert early_reads_of_products(asm) == ["2: v_accvgpr_read_b32 v9, a15"]
    asm = asm.replace("\ts_cbranch", "\ts_nop 15\n\ts_cbranch")
    assert early_reads_of_products(asm) == []


def test_a_jump_is_followed():
    asm = PRODUCT + "\ts_branch LBB0_2\n\tv_mov_b32 v9, a1\nLBB0_2:\n\tglobal_store_dwordx4 v[0:1], a[0:3], off\n"
    assert early_reads_of_products(asm) == ["5: global_store_dwordx4 v[0:1], a[0:3], off"]
