"""What moe_layer_few refuses, before anything is enqueued (no GPU)."""
from paper_2506_12417_amd import binding as B

FAKE = 0x1000


def call(x=FAKE, T=4, d=64, F=64, E=8, k=2, act=B.MOE_RELU, dt=B.MOE_BF16, w_gate=FAKE, norm2=FAKE, bias=None, w_in=FAKE, w_out=FAKE, shared_F=0,
         s_w_in=None, s_w_out=None, idx=FAKE, gate=FAKE, ws=FAKE, ws_bytes=1 << 30, y=FAKE, y_dt=B.MOE_F32):
    try:
        B.moe_layer_few(x, T, d, F, E, k, act, dt, 0, w_gate, norm2, bias, w_in, w_out, shared_F, s_w_in, s_w_out, idx, gate, ws, ws_bytes, y, y_dt, 0)
    except B.MoeError as e:
        assert str(e) and B.moe_last_error()
        return e.status
    return B.MOE_OK


def test_sizes():
    for bad in (dict(T=-1), dict(d=0), dict(F=0), dict(E=0), dict(k=0), dict(k=9, E=8), dict(shared_F=-64)):
        assert call(**bad) == B.MOE_ERR_ARG, bad
    for bad in (dict(T=B.MOE_FEW_MAX_T + 1), dict(E=B.MOE_MAX_EXPERTS + 1), dict(E=32, k=B.MOE_MAX_TOPK + 1), dict(d=96), dict(F=32), dict(shared_F=8),
                dict(act=5), dict(dt=7), dict(y_dt=7), dict(F=1 << 27), dict(d=1 << 27), dict(shared_F=1 << 27, s_w_in=FAKE, s_w_out=FAKE)):
        assert call(**bad) == B.MOE_ERR_UNSUPPORTED, bad


def test_pointers():
    for bad in (dict(x=None), dict(w_gate=None), dict(norm2=None), dict(w_in=None), dict(w_out=None), dict(idx=None), dict(gate=None), dict(y=None),
                dict(shared_F=64)):
        assert call(**bad) == B.MOE_ERR_ARG, bad
    for bad in (dict(x=FAKE + 8), dict(w_gate=FAKE + 2), dict(ws=FAKE + 4)):
        assert call(**bad) == B.MOE_ERR_UNSUPPORTED, bad
    assert call(T=0, x=None, w_gate=None, norm2=None, w_in=None, w_out=None, idx=None, gate=None, ws=None, ws_bytes=0, y=None) == B.MOE_OK


def test_workspace():
    need = B.moe_layer_few_workspace(5, 192, 3, 128, B.MOE_BF16)
    assert need == 5 * (3 * 192 + 128) * 2 and B.moe_layer_few_workspace(5, 192, 3, 128, B.MOE_F32) == 2 * need
    assert call(T=5, F=192, k=3, shared_F=128, s_w_in=FAKE, s_w_out=FAKE, ws_bytes=need - 1) == B.MOE_ERR_WORKSPACE
    assert call(ws=None) == B.MOE_ERR_WORKSPACE
    assert B.moe_layer_few_workspace(-1, 64, 1, 0, 0) == 0 and B.moe_layer_few_workspace(1, 64, 1, 0, 9) == 0


def test_rows_that_offsets_do_not_reach():
    """The first width past each limit is refused and the last one inside passes on to the workspace check: 40 rows of a first matrix with
    SwiGLU (its own or the shared expert's) or 16 without, 16 of a second one, are less than 2 GiB."""
    def first_past(rows, es):
        n = -(-2 ** 31 // (rows * es))
        return -(-n // 64) * 64

    for dt, es in ((B.MOE_BF16, 2), (B.MOE_F32, 4)):
        one = dict(T=1, E=1, k=1, dt=dt, ws_bytes=0)
        shared = dict(shared_F=64, s_w_in=FAKE, s_w_out=FAKE)
        for rows, size, kw in ((40, "d", dict(act=B.MOE_SWIGLU)), (40, "d", shared), (16, "d", dict(act=B.MOE_RELU)), (16, "F", {}), (16, "F", dict(act=B.MOE_SWIGLU)),
                               (16, "shared_F", shared)):
            n = first_past(rows, es)
            assert call(**{**one, **kw, size: n}) == B.MOE_ERR_UNSUPPORTED, (dt, size, kw, n)
            assert call(**{**one, **kw, size: n - 64}) == B.MOE_ERR_WORKSPACE, (dt, size, kw, n)
    assert call(T=1, E=1, k=1, d=1 << 26, act=B.MOE_SWIGLU, ws_bytes=0) == B.MOE_ERR_UNSUPPORTED     # (32 rows of it are 2^32 bytes)


def test_layers_know_what_is_refused():
    """MoELayer.few_ok agrees with the library (tensors without memory: only sizes count)."""
    from paper_2506_12417_amd.layer import MoELayer
    for T, d, F, act in ((1, 64, 64, "relu"), (64, 128, 192, "swiglu"), (65, 64, 64, "relu"), (1, 96, 64, "relu"), (1, 64, 32, "relu"),
                         (1, 1 << 26, 64, "swiglu"), (1, 1 << 25, 64, "relu"), (1, 1 << 25, 64, "swiglu"), (1, 64, 1 << 26, "relu"),
                         (1, 64, (1 << 26) - 64, "relu"), (64, 64, 1 << 24, "relu")):
        L = MoELayer(T, d, F, 1, 1, act, "bf16", 0, device="meta")
        status = call(T=T, d=d, F=F, E=1, k=1, act=B.MOE_SWIGLU if act == "swiglu" else B.MOE_RELU, ws_bytes=0)
        assert L.few_ok == (status == B.MOE_ERR_WORKSPACE) and (L.few_ok or status == B.MOE_ERR_UNSUPPORTED), (T, d, F, act, status)
