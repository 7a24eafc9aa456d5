"""The check of wait states around products written as inline assembly: on listings with planted mistakes, and on the library as it is built."""
import os

import pytest

from paper_2605_10501_amd import binding as B
from paper_2605_10501_amd import mfma_check as M

PRODUCT = "v_mfma_scale_f32_16x16x128_f8f6f4 a[0:3], v[0:7], v[8:15], a[0:3], v16, v17 op_sel:[0,0,0] op_sel_hi:[0,0,0]"
OTHER = "v_mfma_scale_f32_16x16x128_f8f6f4 a[4:7], v[0:7], v[8:15], a[4:7], v16, v17 op_sel:[0,0,0] op_sel_hi:[0,0,0]"


def kernel(*lines):
    """A listing in llvm-objdump's form, four bytes an instruction; "branch k" jumps to line k."""
    out = ["0000000000001000 <kernel>:"]
    for i, l in enumerate([*lines, "s_endpgm"]):
        op, _, to = l.partition(" -> ")
        out.append(f"\t{op}   // {0x1000 + 4 * i:012X}:" + (f" BF850001 <kernel+0x{4 * int(to):x}>" if to else ""))
    return M.parse("\n".join(out))["kernel"]


def bad(*lines):
    return [(o.text, d) for _, o, d in M.hazards(kernel(*lines))]


def test_operands_of_vector_instructions_need_two_states():
    for write in ("v_mov_b32_e32 v0, v30", "v_and_b32_e32 v16, 0xff, v17", "v_lshrrev_b32_e32 v17, 8, v40", "v_accvgpr_write_b32 a2, v30",
                  "v_accvgpr_read_b32 v15, a9", "v_pk_mul_f32 v[6:7], v[20:21], v[22:23]", "v_permlane32_swap_b32_e32 v40, v8"):
        assert bad(write, PRODUCT) == [(write, 0)]
        assert bad(write, "s_nop 0", PRODUCT) == [(write, 1)] and bad(write, "s_add_u32 s0, s1, s2", PRODUCT) == [(write, 1)]
        assert not bad(write, "s_nop 1", PRODUCT) and not bad(write, "s_nop 0", "ds_read_b128 v[50:53], v60", PRODUCT)
    for fine in ("v_mov_b32_e32 v18, v0", "ds_read_b128 v[0:3], v60", "v_cmp_eq_u32_e32 vcc, v0, v1", "s_mov_b32 s0, 1", OTHER):
        assert not bad(fine, PRODUCT), fine


def test_a_written_exec_needs_four_states():
    for write in ("s_mov_b64 exec, s[0:1]", "s_and_saveexec_b64 s[0:1], vcc", "v_cmpx_gt_u32_e32 v1, v2", "s_or_b64 exec, exec, s[0:1]"):
        assert bad(write, "s_nop 2", PRODUCT) == [(write, 3)] and not bad(write, "s_nop 3", PRODUCT)


def test_sums_are_read_late():
    for read in ("v_accvgpr_read_b32 v30, a3", "global_store_dwordx4 v[60:61], a[0:3], off", "v_add_f32_e32 v30, a0, v31", "ds_write_b128 v60, a[0:3]"):
        assert [d for t, d in bad(PRODUCT, read)] == [0] and [d for t, d in bad(PRODUCT, "s_nop 14", read)] == [15]
        assert not bad(PRODUCT, "s_nop 15", read)
    assert not bad(PRODUCT, "v_accvgpr_read_b32 v30, a4", "global_store_dwordx4 v[60:61], v[0:3], off") and not bad(PRODUCT, PRODUCT)


def test_paths_go_through_branches():
    # a loop whose last instruction writes what its first one reads
    assert bad(PRODUCT, "s_nop 7", "v_mov_b32_e32 v0, v30", "s_cbranch_scc1 65532 -> 0") == [("v_mov_b32_e32 v0, v30", 1)]
    assert not bad(PRODUCT, "s_nop 7", "v_mov_b32_e32 v0, v30", "s_nop 0", "s_cbranch_scc1 65531 -> 0")
    # around a wait, which then counts for nothing
    assert bad("v_mov_b32_e32 v0, v30", "s_cbranch_scc1 1 -> 3", "s_nop 7", PRODUCT) == [("v_mov_b32_e32 v0, v30", 1)]
    # an instruction behind an unconditional branch does not follow it
    assert not bad("s_branch 1 -> 2", "v_mov_b32_e32 v0, v30", "s_nop 1", PRODUCT) and not bad(PRODUCT, "s_branch 1 -> 3", "v_accvgpr_read_b32 v1, a0", "s_nop 0")
    # behind the loop the sums of its last trip are as young as those of the branch
    assert [d for _, d in bad(PRODUCT, "s_cbranch_scc1 65534 -> 0", "s_nop 13", "v_accvgpr_read_b32 v30, a0")] == [15]


@pytest.mark.skipif(not os.path.exists(M.OBJDUMP), reason="needs the ROCm tools")
def test_the_library_keeps_its_distances():
    count = M.check(B.LIB_PATH, "gemm_fp8_big_kernel")
    # 256 x 256: 128 products for two K tiles, 256 x 192: 96; whole K tiles and a rest, the first with SwiGLU too
    assert sorted(count.values()) == [96, 96, 128, 128, 128, 128]
    with pytest.raises(RuntimeError, match="no kernel named"):
        M.check(B.LIB_PATH, "no_such_kernel")
