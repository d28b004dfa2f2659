"""What the norms' entry points refuse, before anything is enqueued (no GPU)."""
import pytest

from paper_2506_12417_amd import binding as B

FAKE = 0x1000
ODD = 0x1002


def status(fn, *args):
    try:
        fn(*args)
    except B.MoeError as e:
        assert str(e) and B.moe_last_error()
        return e.status
    return B.MOE_OK


def norm(x=FAKE, x_dt=B.MOE_BF16, w=None, b=None, T=4, d=64, kind=B.MOE_NORM_RMS, eps=1e-5, u=FAKE, u_dt=B.MOE_BF16):
    return status(B.moe_norm, x, x_dt, w, b, T, d, kind, eps, u, u_dt, None, 0)


def norm_back(du=FAKE, x=FAKE, stats=FAKE, T=4, d=64, kind=B.MOE_NORM_RMS, dx=FAKE, dw=None, db=None, ws=None, ws_bytes=0, dt=B.MOE_BF16):
    return status(B.moe_norm_backward, du, dt, x, dt, None, stats, T, d, kind, None, dx, dw, db, ws, ws_bytes, 0)


def end(v=FAKE, h=FAKE, T=4, d=64, post=B.MOE_NORM_RMS, post_eps=1e-5, post_w=None, gate=None, gate_rows=0, nxt=B.MOE_NORM_RMS, next_eps=1e-5,
        next_w=None, y=FAKE, u=FAKE, dts=(B.MOE_BF16,) * 3):
    return status(B.moe_block_end, v, dts[0], h, dts[1], T, d, post, post_eps, post_w, None, gate, gate_rows, 1.0, nxt, next_eps, next_w, None, y, u,
                  dts[2], None, 0)


def rows(y_perm=FAKE, inv=FAKE, k=2, h=FAKE, T=4, d=64, u=FAKE, gate=None, gate_rows=0, dt=B.MOE_BF16):
    return status(B.moe_block_end_rows, y_perm, inv, None, None, k, h, dt, T, d, B.MOE_NORM_NONE, 0.0, None, None, gate, gate_rows, 1.0,
                  B.MOE_NORM_RMS, 1e-5, None, None, FAKE, u, dt, 0)


def end_back(dy=FAKE, du=FAKE, v=FAKE, h=FAKE, T=4, d=64, post=B.MOE_NORM_RMS, gate=None, gate_rows=0, nxt=B.MOE_NORM_RMS, stats=FAKE,
             dpost_w=None, dgate=None, dnext_w=None, ws=None, ws_bytes=0, dt=B.MOE_BF16):
    return status(B.moe_block_end_backward, dy, du, dt, v, dt, h, dt, T, d, post, None, None, gate, gate_rows, 1.0, nxt, None, stats, FAKE, FAKE,
                  dpost_w, None, dgate, dnext_w, None, ws, ws_bytes, 0)


@pytest.mark.parametrize("call", [norm, norm_back, end, rows, end_back])
def test_shapes_and_types(call):
    assert call(T=-1) == B.MOE_ERR_ARG
    assert call(d=0) == B.MOE_ERR_ARG
    assert call(d=B.MOE_NORM_MAX_D + 8) == B.MOE_ERR_UNSUPPORTED
    assert call(d=B.MOE_NORM_ANY_D + 1) == B.MOE_ERR_UNSUPPORTED           # (beyond it only multiples of 8)
    bad = {"dts": (7, 0, 0)} if call is end else {"x_dt": 7} if call is norm else {"dt": 7}
    assert call(**bad) == B.MOE_ERR_UNSUPPORTED


@pytest.mark.parametrize("call", [norm, norm_back, end, rows, end_back])
def test_more_rows_than_an_int_can_step_over(call):
    assert call(T=2 ** 31 - 1) == B.MOE_ERR_UNSUPPORTED and "T=" in str(B.moe_last_error())


def test_long_rows_want_aligned_pointers():
    assert norm(d=8192, x=ODD) == B.MOE_ERR_UNSUPPORTED
    assert end(d=8192, v=ODD) == B.MOE_ERR_UNSUPPORTED
    assert norm_back(d=8192, dx=ODD) == B.MOE_ERR_UNSUPPORTED


def test_norm_arguments():
    assert norm(kind=B.MOE_NORM_NONE) == B.MOE_ERR_ARG and norm(kind=3) == B.MOE_ERR_ARG
    assert norm(eps=-1.0) == B.MOE_ERR_ARG and norm(eps=float("nan")) == B.MOE_ERR_ARG
    assert norm(x=None) == B.MOE_ERR_ARG and norm(u=None) == B.MOE_ERR_ARG
    assert norm(T=0, x=None, u=None) == B.MOE_OK
    for a in ("du", "x", "stats"):
        assert norm_back(**{a: None}) == B.MOE_ERR_ARG
    need = B.moe_workspace_bytes(B.MOE_OP_NORM_BACKWARD, 4, 64, 0, 0, 0, 0)
    assert need > 0
    assert norm_back(dw=FAKE, db=FAKE, ws=FAKE, ws_bytes=need - 1) == B.MOE_ERR_WORKSPACE
    assert norm_back(dw=FAKE, ws=None, ws_bytes=need) == B.MOE_ERR_WORKSPACE


def test_block_end_arguments():
    N = B.MOE_NORM_NONE
    assert end(post=3) == B.MOE_ERR_ARG and end(nxt=-1) == B.MOE_ERR_ARG
    assert end(post_eps=-1.0) == B.MOE_ERR_ARG and end(next_eps=-1.0) == B.MOE_ERR_ARG
    assert end(post=N, post_w=FAKE) == B.MOE_ERR_ARG and end(nxt=N, next_w=FAKE, u=None) == B.MOE_ERR_ARG
    assert end(gate=FAKE, gate_rows=2) == B.MOE_ERR_ARG and end(gate=None, gate_rows=1) == B.MOE_ERR_ARG and end(gate=FAKE) == B.MOE_ERR_ARG
    for a in ("v", "h", "y", "u"):
        assert end(**{a: None}) == B.MOE_ERR_ARG
    assert end(T=0, v=None, h=None, y=None, u=None) == B.MOE_OK
    assert rows(k=0) == B.MOE_ERR_ARG
    for a in ("y_perm", "inv", "h", "u"):
        assert rows(**{a: None}) == B.MOE_ERR_ARG
    assert rows(gate=FAKE, gate_rows=3) == B.MOE_ERR_ARG


def test_block_end_backward_arguments():
    N = B.MOE_NORM_NONE
    for a in ("v", "h", "stats"):
        assert end_back(**{a: None}) == B.MOE_ERR_ARG
    assert end_back(dy=None, du=None) == B.MOE_ERR_ARG
    assert end_back(post=N, dpost_w=FAKE) == B.MOE_ERR_ARG
    assert end_back(nxt=N) == B.MOE_ERR_ARG                                # du without a next norm
    assert end_back(du=None, dnext_w=FAKE) == B.MOE_ERR_ARG
    assert end_back(dgate=FAKE) == B.MOE_ERR_ARG
    need = B.moe_workspace_bytes(B.MOE_OP_BLOCK_END_BACKWARD, 4, 64, 0, 0, 0, 0)
    assert end_back(dpost_w=FAKE, ws=FAKE, ws_bytes=need // 5 - 1) == B.MOE_ERR_WORKSPACE
    assert end_back(gate=FAKE, gate_rows=1, dgate=FAKE) == B.MOE_ERR_WORKSPACE


def test_no_tokens_have_no_gate_gradient():
    """A gate for every token of none: dgate has no rows, so that nothing is enqueued, let alone written there (d zeros were)."""
    none = dict(T=0, dy=None, du=None, v=None, h=None, stats=None, ws=None, ws_bytes=0)
    assert end_back(**none, gate=FAKE, gate_rows=0, dgate=FAKE) == B.MOE_OK


def test_workspace_sizes():
    for op in (B.MOE_OP_NORM_BACKWARD, B.MOE_OP_BLOCK_END_BACKWARD):
        ask = lambda T, d: B.moe_workspace_bytes(op, T, d, 0, 0, 0, 0)    # noqa: E731
        assert ask(-1, 64) == 0 and ask(4, 0) == 0 and ask(4, B.MOE_NORM_MAX_D + 1) == 0
        per = 2 if op == B.MOE_OP_NORM_BACKWARD else 5
        for T, d in ((1, 64), (5000, 64), (5000, 2048), (100000, 8192)):
            assert ask(T, d) % (per * 4 * d) == 0 and ask(T, d) <= 1024 * per * 4 * d


def test_strided_tensors_are_refused():
    import torch
    x = torch.zeros((4, 128), dtype=torch.bfloat16)
    with pytest.raises(B.MoeError) as e:
        B.moe_norm(x[:, :64], B.MOE_BF16, None, None, 4, 64, B.MOE_NORM_RMS, 1e-5, FAKE, B.MOE_BF16, None, 0)
    assert e.value.status == B.MOE_ERR_UNSUPPORTED
    with pytest.raises(B.MoeError):
        B.moe_block_end(x.t(), B.MOE_BF16, FAKE, B.MOE_BF16, 4, 64, 0, 0.0, None, None, None, 0, 1.0, 0, 0.0, None, None, FAKE, None, B.MOE_BF16, None, 0)
