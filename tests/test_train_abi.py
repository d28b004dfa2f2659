"""What the training step's entry points refuse, before anything is enqueued (no GPU)."""
import pytest
import torch

from paper_2506_12417_amd import binding as B
from test_norm_abi import FAKE, ODD, status

F32, BF16 = B.MOE_F32, B.MOE_BF16


def rows(x=FAKE, dt=BF16, rows=4, n=64, q=FAKE, scale=FAKE):
    return status(B.moe_keep_rows, x, dt, rows, n, q, scale, 0)


def restore(x=FAKE, dt=BF16, rows=4, n=64, q=FAKE, scale=FAKE):
    return status(B.moe_keep_restore, q, scale, rows, n, x, dt, 0)


def keep(x=FAKE, T=4, d=64, F=64, E=2, k=1, act=B.MOE_RELU, dt=BF16, w=FAKE, offsets=FAKE, perm=FAKE, h=FAKE, q=FAKE, scale=FAKE):
    return status(B.moe_grouped_ffn_keep, x, T, d, F, E, k, act, dt, w, offsets, perm, h, q, scale, 0)


def back(dy=FAKE, dy_dt=BF16, x=FAKE, T=4, d=64, F=64, E=2, k=1, act=B.MOE_RELU, dt=BF16, w_a=FAKE, w_b=None, w_o=FAKE, offsets=FAKE, perm=FAKE, inv=FAKE,
         gate=None, q=FAKE, scale=FAKE, dx=FAKE, dgate=FAKE, dw_a=FAKE, dw_b=None, dw_o=FAKE, dw_dt=BF16, acc=0, ws=FAKE, ws_bytes=1 << 20):
    return status(B.moe_grouped_ffn_backward, dy, dy_dt, x, T, d, F, E, k, act, dt, w_a, w_b, w_o, offsets, perm, inv, gate, q, scale, dx, dgate, dw_a, dw_b,
                  dw_o, dw_dt, acc, ws, ws_bytes, 0)


def combine(dy=FAKE, dt=BF16, y_perm=FAKE, inv=FAKE, T=4, d=64, k=2, to=FAKE, to_dt=BF16, dgate=FAKE):
    return status(B.moe_unpermute_combine_backward, dy, dt, y_perm, inv, None, T, d, k, to, to_dt, dgate, 0)


def permute(rows=FAKE, inv=FAKE, T=4, d=64, k=2, add=None, dx=FAKE, dt=BF16):
    return status(B.moe_permute_backward, rows, inv, T, d, k, add, dx, dt, 0)


def route(dgate=FAKE, gate=FAKE, idx=FAKE, logits=FAKE, x=FAKE, w=FAKE, T=4, d=64, E=8, k=2, renorm=0, dt=BF16, dl=FAKE, add=None, dx=FAKE, dw=FAKE, db=FAKE,
          ws=FAKE, ws_bytes=1 << 20):
    return status(B.moe_route_topk_backward, dgate, gate, idx, logits, None, x, w, T, d, E, k, renorm, dt, dl, add, dx, dw, db, ws, ws_bytes, 0)


@pytest.mark.parametrize("call", [keep, back, combine, permute, route])
def test_shapes(call):
    assert call(T=-1) == B.MOE_ERR_ARG and call(d=0) == B.MOE_ERR_ARG and call(k=0) == B.MOE_ERR_ARG
    assert call(dt=7) == B.MOE_ERR_UNSUPPORTED
    assert call(T=2 ** 31 - 1, k=2) == B.MOE_ERR_UNSUPPORTED


@pytest.mark.parametrize("call", [keep, back])
def test_ffn_shapes(call):
    assert call(F=0) == B.MOE_ERR_ARG and call(E=0) == B.MOE_ERR_ARG
    assert call(d=96) == B.MOE_ERR_UNSUPPORTED and call(F=100) == B.MOE_ERR_UNSUPPORTED
    assert call(E=B.MOE_MAX_EXPERTS + 1) == B.MOE_ERR_UNSUPPORTED and call(act=2) == B.MOE_ERR_UNSUPPORTED and call(dt=F32) == B.MOE_ERR_UNSUPPORTED
    assert call(T=2 ** 26, d=64) == B.MOE_ERR_UNSUPPORTED                      # x of 8 GiB
    assert call(F=2 ** 22) == B.MOE_ERR_UNSUPPORTED


def test_rows_arguments():
    for call in (rows, restore):
        assert call(rows=-1) == B.MOE_ERR_ARG and call(n=0) == B.MOE_ERR_ARG and call(dt=2) == B.MOE_ERR_UNSUPPORTED
        assert call(rows=0, x=None, q=None, scale=None) == B.MOE_OK
        for a in ("x", "q", "scale"):
            assert call(**{a: None}) == B.MOE_ERR_ARG
        assert call(rows=2 ** 40, n=64) == B.MOE_ERR_UNSUPPORTED and call(rows=2 ** 39, n=4096) == B.MOE_ERR_UNSUPPORTED
        assert call(x=ODD + 1) == B.MOE_ERR_UNSUPPORTED and call(x=ODD, dt=F32) == B.MOE_ERR_UNSUPPORTED and call(scale=ODD) == B.MOE_ERR_UNSUPPORTED


def test_keep_arguments():
    assert keep(T=0, x=None, w=None, offsets=None, perm=None, h=None, q=None, scale=None) == B.MOE_OK
    for a in ("x", "w", "offsets", "perm", "h", "q", "scale"):
        assert keep(**{a: None}) == B.MOE_ERR_ARG
    for a in ("x", "h", "q"):
        assert keep(**{a: ODD}) == B.MOE_ERR_UNSUPPORTED


def test_backward_arguments():
    for a in ("dy", "x", "w_o", "w_a", "offsets", "perm", "inv", "q", "scale"):
        assert back(**{a: None}) == B.MOE_ERR_ARG
    assert back(dw_a=None) == B.MOE_ERR_ARG and back(dw_o=None) == B.MOE_ERR_ARG and back(dw_b=FAKE) == B.MOE_ERR_ARG and back(w_b=FAKE) == B.MOE_ERR_ARG
    sw = dict(act=B.MOE_SWIGLU, w_b=FAKE, dw_b=FAKE)
    assert back(**dict(sw, w_b=None)) == B.MOE_ERR_ARG and back(**dict(sw, dw_b=None)) == B.MOE_ERR_ARG
    for a in ("dy", "x", "w_a", "w_o", "q", "dx", "dw_a", "dw_o", "ws"):
        assert back(**{a: FAKE + 8}) == B.MOE_ERR_UNSUPPORTED
    assert back(dy_dt=5) == B.MOE_ERR_UNSUPPORTED and back(dw_dt=5) == B.MOE_ERR_UNSUPPORTED
    assert back(ws=None) == B.MOE_ERR_WORKSPACE
    need = B.moe_workspace_bytes(B.MOE_OP_FFN_BACKWARD, 4, 64, 64, 2, 1, BF16)
    assert back(**sw, dy_dt=F32, ws_bytes=need - 1) == B.MOE_ERR_WORKSPACE


def test_combine_and_permute_arguments():
    assert combine(T=0, dy=None, y_perm=None, inv=None, to=None, dgate=None) == B.MOE_OK
    assert combine(to=None, dgate=None) == B.MOE_ERR_ARG and combine(y_perm=None) == B.MOE_ERR_ARG
    for a in ("dy", "inv"):
        assert combine(**{a: None}) == B.MOE_ERR_ARG
    assert combine(to_dt=9) == B.MOE_ERR_UNSUPPORTED
    assert permute(T=0, rows=None, inv=None, dx=None) == B.MOE_OK
    for a in ("rows", "inv", "dx"):
        assert permute(**{a: None}) == B.MOE_ERR_ARG
    # more threads than a launch has
    assert combine(T=2 ** 26, k=1) == B.MOE_ERR_UNSUPPORTED and permute(T=2 ** 26, k=1) == B.MOE_ERR_UNSUPPORTED and permute(T=2 ** 20, d=2 ** 16) == B.MOE_ERR_UNSUPPORTED
    assert combine(T=1, d=2 ** 29) == B.MOE_ERR_UNSUPPORTED
    assert rows(rows=2 ** 29, n=64) == B.MOE_ERR_UNSUPPORTED and restore(rows=2 ** 23, n=4096) == B.MOE_ERR_UNSUPPORTED


def test_route_arguments():
    assert route(T=0, dgate=None, gate=None, idx=None, logits=None, x=None, w=None, dl=None, dx=None, dw=None, db=None, ws=None) == B.MOE_OK
    for a in ("dgate", "gate", "idx", "logits", "x", "w", "dl"):
        assert route(**{a: None}) == B.MOE_ERR_ARG
    assert route(k=9, E=16) == B.MOE_ERR_UNSUPPORTED and route(k=9) == B.MOE_ERR_ARG and route(d=60) == B.MOE_ERR_UNSUPPORTED
    assert route(E=B.MOE_MAX_EXPERTS + 1) == B.MOE_ERR_UNSUPPORTED and route(dx=FAKE + 4) == B.MOE_ERR_UNSUPPORTED
    assert route(T=64 * 65535 + 1) == B.MOE_ERR_UNSUPPORTED and route(d=2 ** 20 + 8) == B.MOE_ERR_UNSUPPORTED and route(x=FAKE + 8) == B.MOE_ERR_UNSUPPORTED
    assert route(ws=None) == B.MOE_ERR_WORKSPACE
    assert route(ws_bytes=B.moe_workspace_bytes(B.MOE_OP_ROUTE_BACKWARD, 4, 64, 0, 8, 0, BF16) - 1) == B.MOE_ERR_WORKSPACE


def test_workspace_sizes():
    ask = lambda *a: B.moe_workspace_bytes(*a, BF16)     # noqa: E731
    assert ask(B.MOE_OP_FFN_BACKWARD, -1, 64, 64, 2, 1) == 0 and ask(B.MOE_OP_ROUTE_BACKWARD, 0, 64, 0, 2, 1) == 0
    A, F, T, d = 32768, 1408, 8192, 2048
    assert A * F * 6 <= ask(B.MOE_OP_FFN_BACKWARD, T, d, F, 60, 4) <= A * F * 6 + T * d * 2 + A * F // 16
    assert ask(B.MOE_OP_ROUTE_BACKWARD, T, d, 0, 60, 4) < 64 << 20


def test_strided_tensors_are_refused():
    t = torch.zeros((64, 128), dtype=torch.bfloat16)[:, :64]
    for fn, args in ((B.moe_keep_rows, (t, BF16, 64, 64, FAKE, FAKE, 0)), (B.moe_permute_backward, (FAKE, FAKE, 64, 64, 1, None, t, BF16, 0)),
                     (B.moe_unpermute_combine_backward, (t, BF16, FAKE, FAKE, None, 64, 64, 1, FAKE, BF16, FAKE, 0)),
                     (B.moe_grouped_ffn_keep, (t, 64, 64, 64, 2, 1, B.MOE_RELU, BF16, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0))):
        assert status(fn, *args) == B.MOE_ERR_UNSUPPORTED


def test_layers_that_do_not_train():
    from paper_2506_12417_amd.layer import MoELayer
    with pytest.raises(AssertionError):
        MoELayer(4, 64, 64, 2, 1, "relu", "f32", 0, device="cpu", train=True)


def test_build_checks_the_hand_written_loads_and_stores():
    """build.check_training_kernels: M0 belongs to the loads to LDS, whose three instructions stay together, and a store's registers live on."""
    import os
    from paper_2506_12417_amd import build as b
    load = "\ts_add_u32 m0, s4, 0x1000\n\tv_add_u32_e64 v1, v2, s5 clamp\n\tbuffer_load_dwordx4 v1, s[0:3], s6 offen lds\n"
    small = "\ts_mov_b32 m0, s7\n\ts_nop 0\n\tbuffer_load_dword v3, s[8:11], 0 offen lds\n"
    store = "\tbuffer_store_dwordx4 v[4:7], v8, s[0:3], s9 offen\n\ts_nop 1\n"
    text = lambda body: "_ZN1x14gemm_tn_kernelILi0EEEvv: ; @k\n" + body + "\ts_endpgm\n.Lfunc_end0:\n"      # noqa: E731
    assert b.check_training_kernels(text(load + small + ".LBB0_1:\n" + store + load)) == []
    for line in ("s_mov_b32 m0, s1", "v_readlane_b32 s2, v1, m0", "buffer_load_dwordx4 v1, s[0:3], s6 offen lds"):
        assert [c for _, c in b.check_training_kernels(text(load + "\t" + line + "\n" + store))] == [line], line
    for line, n in (("v_mov_b32_e32 v4, 0", 1), ("v_pk_add_f16 v7, v1, v2", 1), ("v_mov_b32_e32 v3, v4", 0), ("v_accvgpr_write_b32 a4, v4", 0), ("v_mov_b64_e32 v[6:7], v[0:1]", 1)):
        assert len(b.check_training_kernels(text(store.replace("\ts_nop 1\n", "\t" + line + "\n\ts_nop 1\n")))) == n, line
    torn = load.replace("\tbuffer", "\tv_mov_b32_e32 v9, 0\n\tbuffer")
    assert len(b.check_training_kernels(text(torn))) == 2
    assert b.check_training_kernels("_Z1av:\n\ts_endpgm\n.Lfunc_end0:\n")          # no such kernel at all: reported
    asm = os.path.join(os.path.dirname(b.LIB), "_build", "ffn_train.s")
    if os.path.exists(asm):          # the assembly of the library that is loaded here
        whole = open(asm).read()
        assert whole.count(" offen lds") > 500 and b.check_training_kernels(whole) == [] and b.check_no_flat_access(whole) == []
