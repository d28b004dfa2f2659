"""build.check_scalar_wait_states: the wait states between a vector instruction's write of a scalar register and its readers, which neither the hardware nor
(for inline assembly) the compiler sees to, counted on hand-made assembly and on the built kernels' (no GPU)."""
import os

import pytest

from paper_2506_12417_amd import build as b

LANE = "\tv_readfirstlane_b32 s7, v1\n"
LOAD = "\tbuffer_load_dwordx4 v2, s[4:7], s9 offen lds\n"


def found(body):
    return [c for _, c in b.check_scalar_wait_states("_Z1kv: ; @k\n" + body + "\ts_endpgm\n.Lfunc_end0:\n")]


@pytest.mark.parametrize("between,enough", [("", 0), ("\ts_nop 3\n", 0), ("\ts_nop 4\n", 1), ("\ts_add_u32 m0, s1, 0x1000\n\tv_add_u32_e64 v2, v3, s2 clamp\n", 0),
                                            ("\ts_add_u32 m0, s1, 0x1000\n\tv_add_u32_e64 v2, v3, s2 clamp\n\ts_nop 2\n", 1), ("\ts_waitcnt vmcnt(0)\n" * 4, 0),
                                            ("\ts_waitcnt vmcnt(0)\n" * 5, 1), ("\ts_mov_b32 s7, 0x20000\n", 1), ("\ts_mov_b32 s8, 0\n", 0)])
def test_memory_instructions(between, enough):
    for write in (LANE, LANE.replace("s7", "s4"), "\tv_readlane_b32 s5, v9, 3\n", "\tv_cmp_gt_i32_e64 s[6:7], v0, v1\n", "\tv_add_co_u32_e64 v5, s[4:5], v6, v7\n"):
        if "s_mov_b32 s7" in between and "s7" not in write:
            continue
        assert (not found(write + between + LOAD)) == bool(enough), (write, between)
    for read in ("global_atomic_add v250, v2, v3, s[6:7] sc0", "buffer_store_dwordx4 v[0:3], v4, s[0:3], s7 offen", "global_load_dword v1, v2, s[6:7]"):
        assert (not found(LANE + between + "\t" + read + "\n")) == bool(enough), read


def test_the_other_readers():
    assert found(LANE + "\tv_add_u32_e64 v1, v2, s7 clamp\n") and not found(LANE + "\ts_nop 1\n\tv_add_u32_e64 v1, v2, s7 clamp\n")
    assert found(LANE + "\ts_nop 2\n\tv_readlane_b32 s1, v2, s7\n") and not found(LANE + "\ts_nop 3\n\tv_readlane_b32 s1, v2, s7\n")
    # scalar instructions wait by themselves; a vector register of the same number is something else
    assert not found(LANE + "\ts_add_u32 s1, s7, s2\n\ts_nop 4\n") and not found(LANE + "\tbuffer_load_dwordx4 v7, s[8:11], 0 offen lds\n")
    assert found("\tv_cmp_eq_u32_e32 vcc, 0, v1\n\tglobal_load_dword v1, v2, vcc\n")


def test_paths():
    """The write at a loop's end, the read at its start; a branch around the wait."""
    loop = ".LBB0_1:\n" + LOAD + "\ts_nop 4\n" + LANE + "%s\ts_cbranch_scc1 .LBB0_1\n"
    assert found(loop % "") and not found(loop % "\ts_nop 3\n")
    around = LANE + "\ts_cbranch_scc1 .LBB0_2\n\ts_nop 4\n.LBB0_2:\n" + LOAD
    assert found(around) and not found(around.replace(".LBB0_2:\n", ".LBB0_2:\n\ts_nop 3\n"))


@pytest.mark.parametrize("name", ["ffn_train.s", "ffn_bf16.s", "ffn_stream.s", "ffn_wide.s", "ffn_rows.s", "ffn_f32.s"])
def test_the_built_kernels(name):
    asm = os.path.join(os.path.dirname(b.LIB), "_build", name)
    if not os.path.exists(asm):
        pytest.skip("no assembly of the library that is loaded here")
    text = open(asm).read()
    assert "v_readfirstlane_b32" in text and b.check_scalar_wait_states(text) == []
