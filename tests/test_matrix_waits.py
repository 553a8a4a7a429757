"""The build's look at its assembly: reads of a matrix instruction's result with too few wait states, along every path."""
import pytest

from paper_2407_01781_amd.matrix_waits import early_reads

MATRIX = "v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]"          # 11 wait states


def _found(*lines):
    body = "\n".join(line if line.startswith(".L") else "\t" + line for line in lines)
    return early_reads(f"kernel:                ; @kernel\n{body}\n\ts_endpgm\n.Lfunc_end0:\n")


@pytest.mark.parametrize("between,early", [([], True), (["s_nop 9"], True), (["s_nop 10"], False), (["s_nop 7", "s_nop 2"], False), (["v_mov_b32_e32 v20, 0"] * 10, True),
                                           (["v_mov_b32_e32 v20, 0"] * 11, False)])
def test_a_straight_line(between, early):
    assert bool(_found(MATRIX, *between, "v_accvgpr_read_b32 v8, a15")) == early


@pytest.mark.parametrize("read", ["v_add_f32_e32 v8, v9, v3", "v_fmac_f32_e32 v3, v8, v9", "global_store_dwordx4 v[10:11], v[0:3], off", "ds_write_b32 v9, v2", "v_cmp_gt_f32_e32 vcc, 0, v1",
                                  "v_max3_f32 v8, |v9|, |v10|, v0", "ds_read_b32 v9, v1"])
def test_every_kind_of_read(read):
    assert _found("v_mfma_f32_16x16x32_f16 v[0:3], v[4:7], v[12:15], 0", read)
    assert not _found("v_mfma_f32_16x16x32_f16 v[0:3], v[4:7], v[12:15], 0", "s_nop 6", read)


@pytest.mark.parametrize("other", ["v_add_f32_e32 v8, v9, v4", "v_mov_b32_e32 v3, v9", "v_mfma_f32_16x16x32_f16 v[0:3], v[4:7], v[12:15], v[0:3]", "s_add_i32 s0, s1, s2"])
def test_what_is_no_read(other):
    assert not _found("v_mfma_f32_16x16x32_f16 v[0:3], v[4:7], v[12:15], 0", other)


def test_the_shorter_of_two_paths():
    """A branch that skips what the wait states of the longer path are made of."""
    long = ["v_mov_b32_e32 v20, 0"] * 8
    assert not _found(MATRIX, "s_nop 2", *long, ".LBB0_1:", "v_accvgpr_read_b32 v8, a0")
    assert _found(MATRIX, "s_cbranch_scc1 .LBB0_1", *long, ".LBB0_1:", "s_nop 2", "v_accvgpr_read_b32 v8, a0")
    assert not _found(MATRIX, "s_cbranch_scc1 .LBB0_1", *long, ".LBB0_1:", "s_nop 9", "v_accvgpr_read_b32 v8, a0")


def test_around_a_loop():
    assert _found("v_mov_b32_e32 v21, 0", ".LBB0_1:", "v_accvgpr_read_b32 v8, a0", "s_nop 15", MATRIX, "s_cbranch_scc1 .LBB0_1")
    assert not _found("v_mov_b32_e32 v21, 0", ".LBB0_1:", "s_nop 15", "v_accvgpr_read_b32 v8, a0", MATRIX, "s_cbranch_scc1 .LBB0_1")


def test_an_instruction_that_it_does_not_know():
    assert "not known" in _found("v_mfma_f32_4x4x4_16b_f16 v[0:3], v[4:5], v[6:7], 0")[0]
