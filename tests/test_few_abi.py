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
