"""The training step's operators against float64: activations kept in 8 bits, the gradients of the experts, the sort, the combine and the router;
a layer and a block that train, eagerly and from a captured graph.  Tolerances are the bounds that train_ref derives."""
import numpy as np
import pytest

import moe_workloads as W
import train_ref as R
from gpu_util import make_layer

pytestmark = pytest.mark.gpu


def _gpu():
    import torch
    from paper_2506_12417_amd import binding as B
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return torch, B, torch.device("cuda:0")


def rounded(torch, a, dtype):
    """numpy -> a device tensor of this type, and its values in float64."""
    t = torch.from_numpy(np.ascontiguousarray(a)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t.to("cuda:0"), t.double().numpy()


def within(name, got, want, bound):
    got = got.double().cpu().numpy().reshape(want.shape)
    off = np.abs(got - want) - bound
    assert not np.isnan(got).any(), name
    assert (off <= 0).all(), "%s: beyond its bound by up to %g at %s" % (name, off.max(), np.unravel_index(off.argmax(), off.shape))


def ints(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).int().to("cuda:0")


# ------------------------------------------------------------------------------------------------ any rows
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 64), (5, 777), (70, 104), (2, 4096), (257, 65), (33, 1408)])
@pytest.mark.parametrize("dtype,odd", [("f32", 0), ("bf16", 0), ("bf16", 1), ("f32", 1)])
def test_keep_rows(rows, n, dtype, odd):
    torch, B, dev = _gpu()
    print("[case] rows", rows, n, dtype, odd, flush=True)
    r = np.random.default_rng(rows + n)
    x, x64 = rounded(torch, r.standard_normal((rows, n)) * np.exp(3 * r.standard_normal((rows, 1))), dtype)
    code, nb = B.dtype_code(x), R.blocks(n)
    hold = torch.empty(rows * n + 1, dtype=x.dtype, device=dev)
    hold[odd:odd + rows * n] = x.reshape(-1)
    q = torch.full((rows * n + 1,), 99, dtype=torch.int8, device=dev)
    scale = torch.empty((rows, nb), device=dev)
    B.moe_keep_rows(hold[odd:], code, rows, n, q[odd:], scale)
    m = R.block_max(x64)
    within("scale", scale, m[:, ::64] / 127, m[:, ::64] / 127 * 3 * R.U32)
    assert int(q[0 if odd else -1]) == 99
    for out_t, u in ((torch.float32, R.U32), (torch.bfloat16, R.U16)):
        out = torch.empty(rows * n + 1, dtype=out_t, device=dev)
        B.moe_keep_restore(q[odd:], scale, rows, n, out[odd:], B.dtype_code(out))
        within("values", out[odd:odd + rows * n], x64, m / 127 * R.KEPT + (np.abs(x64) + m / 127) * u)


def test_keep_rows_special_values():
    torch, B, dev = _gpu()
    x = torch.ones((6, 128), device=dev)
    x[0, 3] = float("nan")
    x[1, 70] = float("inf")
    x[2, :64] = 0.0
    x[3, :64] = 1e-32
    x[4, :64] = torch.where(torch.arange(64, device=dev) % 2 == 0, 3e38, -3e38)
    x[5, :64] = 1e-30
    q, scale, out = torch.empty((6, 128), dtype=torch.int8, device=dev), torch.empty((6, 2), device=dev), torch.empty((6, 128), device=dev)
    B.moe_keep_rows(x, B.MOE_F32, 6, 128, q, scale)
    B.moe_keep_restore(q, scale, 6, 128, out, B.MOE_F32)
    assert out[0, :64].isnan().all() and (out[0, 64:] == 1).all() and out[1, 64:].isnan().all() and (out[1, :64] == 1).all()
    assert (out[2, :64] == 0).all() and (out[3, :64] == 0).all() and (out[2:, 64:] == 1).all()
    for i in (4, 5):
        assert ((out[i, :64] / x[i, :64] - 1).abs() < 1e-6).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("odd", [0, 1])
def test_keep_rows_ties(dtype, odd):
    """127 v / m = n + 1/2 exactly, of values that both types hold: to the even neighbour."""
    torch, B, dev = _gpu()
    n = torch.arange(126, dtype=torch.float64, device=dev).reshape(2, 63)
    v = torch.cat([torch.full((2, 1), 127 / 128, dtype=torch.float64, device=dev), (2 * n + 1) / 256], 1)
    want = torch.cat([torch.full((2, 1), 127.0, dtype=torch.float64, device=dev), torch.round((n + 0.5))], 1)
    assert (want[:, 1:] % 2 == 0).all()
    x = torch.cat([torch.cat([v, -v]) * 2.0 ** e for e in (-99, -3, 0, 1, 128)]).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    assert (x.double()[8:12] == torch.cat([v, -v])).all()
    hold = torch.empty(x.numel() + 1, dtype=x.dtype, device=dev)
    hold[odd:odd + x.numel()] = x.reshape(-1)
    q, scale = torch.empty(x.shape, dtype=torch.int8, device=dev), torch.empty((x.shape[0], 1), device=dev)
    B.moe_keep_rows(hold[odd:], B.dtype_code(x), x.shape[0], 64, q, scale)
    assert (q.double() == torch.cat([want, -want] * 5)).all()


# ------------------------------------------------------------------------------------------------ the experts
SHAPES = [  # T, d, F, E, k, act, kind of routing
    (1, 64, 64, 1, 1, "relu", {}),
    (1, 128, 192, 5, 3, "swiglu", {}),
    (40, 320, 448, 6, 2, "relu", dict(empty=(0, 5))),
    (130, 256, 320, 7, 2, "swiglu", dict(empty=(3,))),
    (300, 192, 128, 3, 1, "swiglu", dict(one=1)),
    (700, 64, 576, 4, 2, "relu", {}),
    (1500, 320, 192, 2, 1, "swiglu", {}),
    (1100, 128, 64, 1, 1, "relu", {}),
    (256, 64, 64, 2, 2, "swiglu", {}),
    (65, 576, 64, 256, 8, "relu", {}),
]


def make_case(torch, T, d, F, E, k, act, how, seed):
    r = np.random.default_rng(seed)
    x = rounded(torch, r.standard_normal((T, d)), "bf16")
    dy = rounded(torch, r.standard_normal((T, d)), "bf16")
    w = {n: rounded(torch, r.standard_normal((E, d, F)) * d ** -0.5, "bf16") for n in ("ab" if act == "swiglu" else "a")}
    w["o"] = rounded(torch, r.standard_normal((E, F, d)) * F ** -0.5, "bf16")
    gate = r.random((T, k)).astype(np.float32)
    return x, dy, w, gate, R.routing(T, k, E, seed, **how)


def pack(torch, B, w, E, d, F, act):
    p = torch.empty((E, 2 * F if act == "swiglu" else F, d), dtype=torch.bfloat16, device="cuda:0")
    B.moe_pack_weights(w["a"][0], w["b"][0] if "b" in w else None, E, d, F, B.MOE_BF16, p)
    return p, p.data_ptr() + torch.arange(E, device="cuda:0") * (p.shape[1] * d * 2)


@pytest.mark.parametrize("T,d,F,E,k,act,how", SHAPES)
def test_grouped_ffn_keep(T, d, F, E, k, act, how):
    torch, B, dev = _gpu()
    print("[case] keep", T, d, F, E, k, act, how, flush=True)
    (x, x64), _, w, _, rt = make_case(torch, T, d, F, E, k, act, how, T + d)
    packed, ptrs = pack(torch, B, w, E, d, F, act)
    A, Z = T * k, packed.shape[1]
    h = torch.full((A + 1, F), 7.0, dtype=torch.float16, device=dev)
    q, scale = torch.full((A + 1, Z), 99, dtype=torch.int8, device=dev), torch.full((A + 1, Z // 64), 7.0, device=dev)
    B.moe_grouped_ffn_keep(x, T, d, F, E, k, getattr(B, "MOE_" + act.upper()), B.MOE_BF16, ptrs, ints(torch, rt["offsets"]), ints(torch, rt["perm"]), h, q, scale)
    z, err = R.first_product(x64, {n: v[1] for n, v in w.items()}, rt, k, act)
    kept = R.restore(q[:A].cpu().numpy(), scale[:A].cpu().numpy())
    m = R.block_max(z) + R.block_max(err)
    assert (np.abs(kept - z) <= err + m / 127 * (R.KEPT if act == "swiglu" else 1.0 + 1e-4)).all()
    if act == "relu":
        assert (kept >= 0).all() and ((kept > 0) >= (z > err)).all() and ((kept > 0) <= (z > -err)).all()
        he = err
    else:
        (g, u), (ge, ue) = np.split(z, 2, 1), np.split(err, 2, 1)
        he = 1.2 * np.abs(u) * ge + np.abs(g) * ue + (8 + 2 * np.abs(g)) * R.U32 * np.abs(g * u)
    hid = R.hidden(z, act)
    within("h", h[:A], hid, he + np.abs(hid) * R.UH + 2.0 ** -25)
    assert (h[A] == 7).all() and (q[A] == 99).all() and (scale[A] == 7).all()


def run_back(torch, B, x, dy, w, gate, rt, q, scale, T, d, F, E, k, act, dw_t=None, dw=None, accumulate=0, dgate=True, dxp=True):
    dev = "cuda:0"
    A = T * k
    like = lambda n: torch.full(tuple(w[n].shape), 5.0, dtype=dw_t, device=dev) if n in w else None     # noqa: E731
    dw = dw if dw is not None else {n: like(n) for n in "abo"}
    dx_perm = torch.full((A + 1, d), 7.0, device=dev) if dxp else None
    dgate_w = torch.empty((T, k), device=dev) if dgate else None
    ws = torch.empty(B.moe_workspace_bytes(B.MOE_OP_FFN_BACKWARD, T, d, F, E, k, B.MOE_BF16), dtype=torch.uint8, device=dev)
    B.moe_grouped_ffn_backward(dy, B.dtype_code(dy), x, T, d, F, E, k, getattr(B, "MOE_" + act.upper()), B.MOE_BF16, w["a"], w.get("b"), w["o"],
                               ints(torch, rt["offsets"]), ints(torch, rt["perm"]), ints(torch, rt["inv"]), gate, q, scale, dx_perm, dgate_w, dw["a"],
                               dw["b"], dw["o"], B.dtype_code(dw["o"]) if dw["o"] is not None else B.MOE_BF16, accumulate, ws, ws.numel())
    return dx_perm, dgate_w, dw


def kept_values(torch, A, Z, act, seed):
    r = np.random.default_rng(seed)
    q = r.integers(-127, 128, (A, Z))
    q[r.random((A, Z)) < 0.05] = 0
    scale = (r.random((A, Z // 64)) * 0.04 + 0.001).astype(np.float32)
    if act == "relu":
        q = np.maximum(q, 0)
    return q.astype(np.int8), scale


@pytest.mark.parametrize("T,d,F,E,k,act,how", SHAPES)
@pytest.mark.parametrize("dw_type", ["bf16", "f32"])
def test_grouped_ffn_backward(T, d, F, E, k, act, how, dw_type):
    torch, B, dev = _gpu()
    print("[case] backward", T, d, F, E, k, act, how, dw_type, flush=True)
    (x, x64), (dy, dy64), w, gate, rt = make_case(torch, T, d, F, E, k, act, how, T + d)
    A = T * k
    q, scale = kept_values(torch, A, 2 * F if act == "swiglu" else F, act, T)
    with_gate = T % 2 == 0
    g64 = gate.astype(np.float64) if with_gate else np.ones((T, k))
    dw_t = torch.bfloat16 if dw_type == "bf16" else torch.float32
    args = (torch, B, x, dy, {n: v[0] for n, v in w.items()}, torch.from_numpy(gate).to(dev) if with_gate else None, rt, torch.from_numpy(q).to(dev),
            torch.from_numpy(scale).to(dev), T, d, F, E, k, act)
    dx_perm, dgate_w, dw = run_back(*args, dw_t=dw_t)
    (dxp, dxe), (dg, dge), ref = R.ffn_backward(x64, dy64, {n: v[1] for n, v in w.items()}, rt, k, g64, R.restore(q, scale), act)
    within("dx_perm", dx_perm[:A], dxp, dxe)
    assert (dx_perm[A] == 7).all()
    within("dgate_w", dgate_w, dg.reshape(T, k), dge.reshape(T, k))
    for n in ref:
        within("dw " + n, dw[n], ref[n][0], ref[n][1] + np.abs(ref[n][0]) * R.unit(dw_type))
    assert dw["b"] is None or act == "swiglu"
    # the same call, the same bits; added to what is there
    again = run_back(*args, dw_t=dw_t)
    assert torch.equal(again[0], dx_perm) and torch.equal(again[1], dgate_w) and all(torch.equal(again[2][n], dw[n]) for n in ref)
    first = {n: dw[n].clone() if dw[n] is not None else None for n in "abo"}
    run_back(*args, dw=dw, accumulate=1, dgate=False, dxp=False)
    for n in ref:
        within("sum " + n, dw[n], 2 * ref[n][0], 2 * ref[n][1] + np.abs(ref[n][0]) * 3.1 * R.unit(dw_type))
        none = torch.from_numpy(rt["counts"] == 0).to(dev)
        assert torch.equal(dw[n][none], first[n][none])


def test_backward_of_an_fp32_gradient_and_without_matrices():
    torch, B, dev = _gpu()
    T, d, F, E, k, act = 90, 192, 128, 5, 2, "swiglu"
    (x, _), (dy, _), w, gate, rt = make_case(torch, T, d, F, E, k, act, {}, 4)
    q, scale = kept_values(torch, T * k, 2 * F, act, 1)
    w = {n: v[0] for n, v in w.items()}
    fine = torch.from_numpy(np.random.default_rng(3).standard_normal((T, d)).astype(np.float32)).to(dev)
    one = lambda g, **kw: run_back(torch, B, x, g, w, torch.from_numpy(gate).to(dev), rt, torch.from_numpy(q).to(dev), torch.from_numpy(scale).to(dev),     # noqa: E731
                                   T, d, F, E, k, act, **kw)
    a, b = one(fine, dw_t=torch.float32), one(fine.bfloat16(), dw_t=torch.float32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and all(torch.equal(a[2][n], b[2][n]) for n in "abo")
    c = one(fine, dw={n: None for n in "abo"})
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


def test_backward_without_tokens():
    torch, B, dev = _gpu()
    dw = {n: torch.full((3, 64, 128) if n != "o" else (3, 128, 64), 5.0, device=dev, dtype=torch.bfloat16) for n in "ao"}
    zero = torch.zeros(4, dtype=torch.int32, device=dev)
    call = lambda acc: B.moe_grouped_ffn_backward(None, B.MOE_BF16, None, 0, 64, 128, 3, 1, B.MOE_RELU, B.MOE_BF16, None, None, None, zero, None, None, None,    # noqa: E731
                                                  None, None, None, None, dw["a"], None, dw["o"], B.MOE_BF16, acc, None, 0)
    call(1)
    assert (dw["a"] == 5).all() and (dw["o"] == 5).all()
    call(0)
    assert not dw["a"].any() and not dw["o"].any()


def test_assignments_without_a_row():
    """Tokens whose logits were NaN: nothing is read or written for them, behind the last row nothing changes."""
    torch, B, dev = _gpu()
    T, d, F, E, k, act = 75, 128, 192, 4, 2, "swiglu"
    (x, x64), (dy, dy64), w, gate, rt = make_case(torch, T, d, F, E, k, act, {}, 8)
    idx = rt["idx"].copy()
    idx[[0, 33, 74]] = E
    rt = R.sort(idx, E)
    n, A = int(rt["offsets"][-1]), T * k
    assert n == A - 6
    perm = dict(rt, perm=np.concatenate([rt["perm"], np.full(A - n, 2 ** 30, np.int32)]))
    packed, ptrs = pack(torch, B, w, E, d, F, act)
    h, q, scale = torch.full((A, F), 7.0, dtype=torch.float16, device=dev), torch.full((A, 2 * F), 99, dtype=torch.int8, device=dev), torch.full((A, F // 32), 7.0, device=dev)
    B.moe_grouped_ffn_keep(x, T, d, F, E, k, B.MOE_SWIGLU, B.MOE_BF16, ptrs, ints(torch, rt["offsets"]), ints(torch, perm["perm"]), h, q, scale)
    assert (h[n:] == 7).all() and (q[n:] == 99).all() and (scale[n:] == 7).all()
    dxp, dgate, dw = run_back(torch, B, x, dy, {m: v[0] for m, v in w.items()}, torch.from_numpy(gate).to(dev), perm, q, scale, T, d, F, E, k, act, dw_t=torch.float32)
    assert (dxp[n:] == 7).all()
    z = R.restore(q[:n].cpu().numpy(), scale[:n].cpu().numpy())
    (want, bound), (dg, dge), ref = R.ffn_backward(x64, dy64, {m: v[1] for m, v in w.items()}, rt, k, gate.astype(np.float64), z, act)
    within("dx_perm", dxp[:n], want, bound)
    within("dgate_w", dgate, dg.reshape(T, k), dge.reshape(T, k))
    assert not dgate[0].any() and not dgate[33].any()
    for m in ref:
        within("dw " + m, dw[m], ref[m][0], ref[m][1] + np.abs(ref[m][0]) * R.U32)


def test_not_a_number_reaches_what_it_takes_part_in():
    torch, B, dev = _gpu()
    T, d, F, E, k = 8, 64, 128, 2, 1
    for act in ("relu", "swiglu"):
        (x, _), (dy, _), w, _, rt = make_case(torch, T, d, F, E, k, act, {}, 9)
        rt = R.sort(np.array([[0]] * 5 + [[1]] * 3, dtype=np.int32), E)
        x[2, 5] = float("nan")
        packed, ptrs = pack(torch, B, w, E, d, F, act)
        Z = packed.shape[1]
        h, q, scale = torch.empty((T, F), dtype=torch.float16, device=dev), torch.empty((T, Z), dtype=torch.int8, device=dev), torch.empty((T, Z // 64), device=dev)
        B.moe_grouped_ffn_keep(x, T, d, F, E, k, getattr(B, "MOE_" + act.upper()), B.MOE_BF16, ptrs, ints(torch, rt["offsets"]), ints(torch, rt["perm"]), h, q, scale)
        assert h[2].isnan().all() and scale[2].isnan().all() and not h[[0, 1, 3, 4, 5, 6, 7]].isnan().any() and scale.isnan().sum() == Z // 64
        dxp, dgate, dw = run_back(torch, B, x, dy, {n: v[0] for n, v in w.items()}, None, rt, q, scale, T, d, F, E, k, act, dw_t=torch.bfloat16)
        others = [0, 1, 3, 4, 5, 6, 7]
        assert dxp[2].isnan().all() and not dxp[others].isnan().any() and dgate[2].isnan().all() and not dgate[others].isnan().any()
        for n in w:
            assert dw[n][0].isnan().any() and not dw[n][1].isnan().any()


def test_kept_values_and_gradients_beyond_2_31_bytes():
    """One expert's rows whose kept values and their gradients take more than a 32-bit offset reaches."""
    torch, B, dev = _gpu()
    T, d, F, E, k = 98304, 64, 14336, 2, 1
    print("[case] long", T, d, F, flush=True)
    gen = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn((T, d), device=dev, generator=gen).bfloat16()
    dy = torch.randn((T, d), device=dev, generator=gen).bfloat16()
    w = {n: (torch.randn((E, d, F) if n != "o" else (E, F, d), device=dev, generator=gen) * 0.1).bfloat16() for n in "abo"}
    n0 = 100
    rt = dict(offsets=np.array([0, n0, T]), perm=np.arange(T), inv=np.arange(T))
    packed, ptrs = pack(torch, B, {n: (v,) for n, v in w.items()}, E, d, F, "swiglu")
    h, q, scale = torch.empty((T, F), dtype=torch.float16, device=dev), torch.empty((T, 2 * F), dtype=torch.int8, device=dev), torch.empty((T, F // 32), device=dev)
    B.moe_grouped_ffn_keep(x, T, d, F, E, k, B.MOE_SWIGLU, B.MOE_BF16, ptrs, ints(torch, rt["offsets"]), ints(torch, rt["perm"]), h, q, scale)
    dw = {n: torch.empty(v.shape, device=dev) for n, v in w.items()}
    dxp, dgate, _ = run_back(torch, B, x, dy, w, None, rt, q, scale, T, d, F, E, k, "swiglu", dw=dw)
    at = [0, n0 - 1, n0, 75000, T - 1]                     # (rows that lie beyond 2^31 bytes of q and 2^32 of its gradient among them)
    X, DY, W64 = x[at].double().cpu().numpy(), dy[at].double().cpu().numpy(), {n: v.double().cpu().numpy() for n, v in w.items()}
    few = R.sort(np.array([[0], [0], [1], [1], [1]], dtype=np.int32), E)
    z, err = R.first_product(X, W64, few, 1, "swiglu")
    kept = R.restore(q[at].cpu().numpy(), scale[at].cpu().numpy())
    assert (np.abs(kept - z) <= err + (R.block_max(z) + R.block_max(err)) / 127 * R.KEPT).all()
    (want, bound), (dg, dge), _ = R.ffn_backward(X, DY, W64, few, 1, np.ones((5, 1)), kept, "swiglu")
    within("dx_perm", dxp[at], want, bound)
    within("dgate_w", dgate[at], dg.reshape(5, 1), dge.reshape(5, 1))
    # some columns of the second expert's gradients, whole sums on the GPU in float64
    cols = slice(F - 64, F)
    zz = (q[n0:, F - 64:F].double() * scale[n0:, F // 64 - 1:F // 64].double(), q[n0:, 2 * F - 64:].double() * scale[n0:, -1:].double())
    s = dy[n0:].double() @ w["o"][1][cols].double().t()
    sig = torch.sigmoid(zz[0])
    dg_ = s * zz[1] * sig * (1 + zz[0] * (1 - sig))
    for name, got, L, Rr in (("a", dw["a"][1][:, cols], x[n0:].double(), dg_), ("o", dw["o"][1][cols].t(), dy[n0:].double(), zz[0] * sig * zz[1])):
        ref, mag = L.t() @ Rr, L.abs().t() @ Rr.abs()
        assert ((got.double() - ref).abs() <= mag * (R.U16 * 1.01 + T * R.U32)).all(), name


# ------------------------------------------------------------------------------------------------ the sort and the combine
@pytest.mark.parametrize("T,d,k", [(1, 1, 1), (3, 8, 8), (50, 777, 3), (70, 520, 4), (9, 2048, 9), (600, 64, 2)])
@pytest.mark.parametrize("dtype,to", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("lost", [False, True])
def test_combine_and_permute_backward(T, d, k, dtype, to, lost):
    torch, B, dev = _gpu()
    print("[case] sort", T, d, k, dtype, to, lost, flush=True)
    r = np.random.default_rng(T + d + k)
    A = T * k
    inv = r.permutation(A).astype(np.int32)
    n = A
    if lost:
        gone = r.random(A) < 0.3
        n = int((~gone).sum())
        inv[~gone] = r.permutation(n)
        inv[gone] = -1
    dy, dy64 = rounded(torch, r.standard_normal((T, d)), dtype)
    yp, yp64 = rounded(torch, r.standard_normal((A, d)), "f32")
    add, add64 = rounded(torch, r.standard_normal((T, d)), "f32")
    gate = r.random((T, k)).astype(np.float32) if T != 50 else None
    to_t = torch.float32 if to == "f32" else torch.bfloat16
    dyp, dgate = torch.full((A + 1, d), 7.0, dtype=to_t, device=dev), torch.empty((T, k), device=dev)
    B.moe_unpermute_combine_backward(dy, B.dtype_code(dy), yp, ints(torch, inv), None if gate is None else torch.from_numpy(gate).to(dev), T, d, k, dyp, B.dtype_code(dyp), dgate)
    on = inv >= 0
    want, tok = np.zeros((n, d)), np.arange(A) // k
    want[inv[on]] = (dy64[tok] * (1.0 if gate is None else gate.astype(np.float64).reshape(-1, 1)))[on]
    within("dy_perm", dyp[:n], want, np.abs(want) * (R.unit(to) + R.U32))
    assert (dyp[n:] == 7).all()
    prod = dy64[tok] * yp64[np.maximum(inv, 0)] * on[:, None]
    within("dgate_w", dgate, prod.sum(1).reshape(T, k), (d + 1) * R.U32 * np.abs(prod).sum(1).reshape(T, k))
    only = torch.full((A + 1, d), 7.0, dtype=to_t, device=dev)
    B.moe_unpermute_combine_backward(dy, B.dtype_code(dy), None, ints(torch, inv), None if gate is None else torch.from_numpy(gate).to(dev), T, d, k, only, B.dtype_code(only), None)
    assert torch.equal(only, dyp)
    for with_add in (True, False):
        dx = torch.empty((T, d), dtype=to_t, device=dev)
        B.moe_permute_backward(yp, ints(torch, inv), T, d, k, add if with_add else None, dx, B.dtype_code(dx))
        rows = (yp64[np.maximum(inv, 0)] * on[:, None]).reshape(T, k, d)
        ref = rows.sum(1) + (add64 if with_add else 0)
        mag = np.abs(rows).sum(1) + (np.abs(add64) if with_add else 0)
        within("dx", dx, ref, (k + 1) * R.U32 * mag + R.unit(to) * (np.abs(ref) + (k + 1) * R.U32 * mag))


def test_permute_backward_in_place():
    torch, B, dev = _gpu()
    rows, add = torch.randn((12, 40), device=dev), torch.randn((4, 40), device=dev)
    inv = torch.randperm(12, device=dev).int()
    dx = torch.empty((4, 40), device=dev)
    B.moe_permute_backward(rows, inv, 4, 40, 3, add, dx, B.MOE_F32)
    B.moe_permute_backward(rows, inv, 4, 40, 3, add, add, B.MOE_F32)
    assert torch.equal(dx, add)


# ------------------------------------------------------------------------------------------------ the router
@pytest.mark.parametrize("T,d,E,k", [(1, 8, 1, 1), (2, 64, 256, 8), (33, 136, 7, 3), (700, 768, 128, 1), (65, 320, 60, 4), (3001, 72, 130, 2)])
@pytest.mark.parametrize("renorm", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_route_backward(T, d, E, k, renorm, dtype):
    torch, B, dev = _gpu()
    print("[case] route", T, d, E, k, renorm, dtype, flush=True)
    r = np.random.default_rng(T + E)
    x, x64 = rounded(torch, r.standard_normal((T, d)), dtype)
    w, w64 = rounded(torch, r.standard_normal((d, E)) * d ** -0.5, dtype)
    idx, gate, logits = torch.empty((T, k), dtype=torch.int32, device=dev), torch.empty((T, k), device=dev), torch.empty((T, E), device=dev)
    B.moe_route_topk(x, w, None, T, d, E, k, renorm, B.dtype_code(x), idx, gate, logits)
    dgate, dg64 = rounded(torch, r.standard_normal((T, k)), "f32")
    extra, extra64 = rounded(torch, 0.1 * r.standard_normal((T, E)), "f32")
    add, add64 = rounded(torch, r.standard_normal((T, d)), "f32")
    ws = torch.empty(B.moe_workspace_bytes(B.MOE_OP_ROUTE_BACKWARD, T, d, 0, E, 0, B.dtype_code(x)), dtype=torch.uint8, device=dev)
    dl, dx, dw, db = torch.empty((T, E), device=dev), torch.empty((T, d), device=dev), torch.empty((d, E), device=dev), torch.empty(E, device=dev)
    run = lambda ex, ad: B.moe_route_topk_backward(dgate, gate, idx, None if renorm else logits, ex, x, w, T, d, E, k, renorm, B.dtype_code(x), dl, ad, dx, dw, db,    # noqa: E731
                                                   ws, ws.numel())
    run(extra, add)
    g64, i64, l64 = gate.double().cpu().numpy(), idx.cpu().numpy(), logits.double().cpu().numpy()
    ref = R.route_backward(l64, i64, g64, dg64, renorm)
    # the gates (k products and sums), the softmax (an exponential of up to |logit| roundings, a sum of E) and its products
    size = (np.abs(g64) * np.abs(dg64)).sum(1, keepdims=True) + np.abs(dg64).max(1, keepdims=True)
    rel = (2 * k + 8 + E + 2 * np.abs(l64 - l64.max(1, keepdims=True))) * R.U32
    p = np.exp(l64 - l64.max(1, keepdims=True))
    p = p / p.sum(1, keepdims=True)
    if renorm:
        p = np.zeros_like(p)
        p[np.arange(T)[:, None], i64] = g64
    err = rel * p * size + (np.abs(ref) + np.abs(extra64)) * R.U32
    within("dlogits", dl, ref + extra64, err)
    own = dl.double().cpu().numpy()                        # (what the sums are made of)
    within("dx", dx, add64 + own @ w64.T, (E + 2) * R.U32 * (np.abs(own) @ np.abs(w64.T) + np.abs(add64)))
    within("dw", dw, x64.T @ own, (T + 2) * R.U32 * (np.abs(x64.T) @ np.abs(own)))
    within("db", db, own.sum(0), (T + 2) * R.U32 * np.abs(own).sum(0))
    both = [t.clone() for t in (dl, dx, dw, db)]
    run(extra, add)
    assert all(torch.equal(a, b) for a, b in zip(both, (dl, dx, dw, db)))
    run(None, None)
    within("plain dlogits", dl, ref, err)
    # each by itself, none of the others touched; added in place
    dl2, db2 = torch.empty_like(dl), torch.empty_like(db)
    B.moe_route_topk_backward(dgate, gate, idx, logits, None, None, None, T, d, E, k, renorm, B.dtype_code(x), dl2, None, None, None, db2, ws, ws.numel())
    assert torch.equal(dl, dl2) and torch.equal(db, db2)
    B.moe_route_topk_backward(dgate, gate, idx, logits, extra, None, w, T, d, E, k, renorm, B.dtype_code(x), dl2, add, add, None, None, None, 0)
    assert torch.equal(add, both[1])


def test_route_backward_special_rows():
    torch, B, dev = _gpu()
    T, d, E, k = 5, 64, 6, 2
    x, w = torch.randn((T, d), device=dev), torch.randn((d, E), device=dev)
    idx = torch.tensor([[0, 1], [6, 6], [2, 5], [-1, 0], [3, 4]], dtype=torch.int32, device=dev)
    logits, gate, dg = torch.randn((T, E), device=dev), torch.rand((T, k), device=dev), torch.randn((T, k), device=dev)
    logits[0, 2] = -float("inf")                           # an expert that is masked
    dl, dx = torch.empty((T, E), device=dev), torch.empty((T, d), device=dev)
    for renorm in (0, 1):
        B.moe_route_topk_backward(dg, gate, idx, logits, None, x, w, T, d, E, k, renorm, B.MOE_F32, dl, None, dx, None, None, None, 0)
        assert dl[[1, 3]].isnan().all() and not dl[[0, 2, 4]].isnan().any() and dl[0, 2] == 0 and dx[[1, 3]].isnan().all() and not dx[[0, 2, 4]].isnan().any()
    dw, db = torch.ones((d, E), device=dev), torch.ones(E, device=dev)
    B.moe_route_topk_backward(None, None, None, None, None, None, None, 0, d, E, k, 0, B.MOE_F32, None, None, None, dw, db, None, 0)
    assert not dw.any() and not db.any()


# ------------------------------------------------------------------------------------------------ a layer and a block that train
def trained_layer(T, d, F, E, k, act, renorm, shared_F=0, seed=1):
    wl = W.MoEWorkload("train", 6, T, d, F, E, k, act, "bf16", renorm, shared_F=shared_F)
    inp = W.make_inputs(wl, seed=seed)
    return make_layer(wl, inp, train=True), make_layer(wl, inp)


LAYERS = [(1, 256, 512, 4, 1, "relu", 0, 0), (90, 320, 192, 6, 2, "swiglu", 1, 128), (300, 256, 512, 8, 1, "relu", 0, 0), (257, 192, 320, 12, 4, "swiglu", 0, 0),
          (129, 128, 64, 5, 2, "swiglu", 1, 64)]


@pytest.mark.parametrize("T,d,F,E,k,act,renorm,shared_F", LAYERS)
def test_layer(T, d, F, E, k, act, renorm, shared_F):
    torch, B, dev = _gpu()
    print("[case] layer", T, d, F, E, k, act, renorm, shared_F, flush=True)
    L, plain = trained_layer(T, d, F, E, k, act, renorm, shared_F)
    r = np.random.default_rng(T)
    x, x64 = rounded(torch, r.standard_normal((T, d)), "bf16")
    dy, _ = rounded(torch, r.standard_normal((T, d)), "f32")
    y = L.forward(x).clone()
    plain.forward(x)
    assert torch.equal(L.expert_idx, plain.expert_idx) and torch.equal(L.gate_w, plain.gate_w)
    w64 = {n: w.double().cpu().numpy() for n, w in L.weight.items() if w is not None}
    rt, gate = R.sort(L.expert_idx.cpu().numpy(), E), L.gate_w.double().cpu().numpy()
    one = R.sort(np.zeros((T, 1), np.int32), 1)
    parts = [({n: w64[n] for n in w64 if len(n) == 1}, rt, k, gate, act, "")] + (
        [({n: w64["s" + n] for n in "abo"}, one, 1, np.ones((T, 1)), "swiglu", "s")] if shared_F else [])
    want, bound = np.zeros((T, d)), np.zeros((T, d))
    for w, t, kk, g, a, _ in parts:
        z, err = R.first_product(x64, w, t, kk, a)
        h = R.hidden(z, a)
        if a == "swiglu":
            (zg, zu), (ge, ue) = np.split(z, 2, 1), np.split(err, 2, 1)
            err = 1.2 * np.abs(zu) * ge + np.abs(zg) * ue + (8 + 2 * np.abs(zg)) * R.U32 * np.abs(zg * zu)
        err = err + R.UH * (np.abs(h) + err) + 2.0 ** -25
        for e in range(len(t["counts"])):
            sl = slice(t["offsets"][e], t["offsets"][e + 1])
            ids, wo = t["perm"][sl], w["o"][e]
            gg = g.reshape(-1)[ids][:, None]
            np.add.at(want, ids // kk, gg * (h[sl] @ wo))
            # (the second matrix in half: values below 2^-14 are off by up to 2^-25)
            off = err[sl] @ np.abs(wo) + np.abs(h[sl]) @ (np.abs(wo) * (h.shape[1] + 12) * R.U32 + 2.0 ** -25)
            np.add.at(bound, ids // kk, gg * off)
    within("y", y, want, bound + 4 * R.U32 * np.abs(want))
    dx = L.backward(dy, x)
    check_gradients(torch, L, parts, x64, dy, dx, None)
    # the same again, and with the experts' gradients added up
    before = {n: t.clone() for n, t in L.grad.items() if t is not None}
    first = dx.clone()
    extra, _ = rounded(torch, 0.1 * r.standard_normal((T, E)), "f32")
    assert torch.equal(L.backward(dy, x), first) and all(torch.equal(before[n], L.grad[n]) for n in before)
    dx = L.backward(dy.bfloat16(), x, extra, accumulate=True)
    check_gradients(torch, L, parts, x64, dy, dx, extra, times=2)


def check_gradients(torch, L, parts, x64, dy, dx, extra, times=1):
    T, d, k = L.T, L.d, L.k
    dy64 = dy.bfloat16().double().cpu().numpy()
    got = lambda t: t.double().cpu().numpy()      # noqa: E731
    dl, wg = got(L.dlogits), got(L.W_g)
    ref = R.route_backward(got(L.logits), L.expert_idx.cpu().numpy(), got(L.gate_w), got(L.dgate_w), L.renorm)
    ex = 0.0 if extra is None else got(extra)
    size = np.abs(got(L.dgate_w)).max(1, keepdims=True) * 2
    within("dlogits", L.dlogits, ref + ex, (L.E + 80) * R.U32 * size + (np.abs(ref) + np.abs(ex)) * R.U32)
    want = dl @ wg.T
    bound = (L.E + 4) * R.U32 * (np.abs(dl) @ np.abs(wg.T))
    for w, t, kk, g, a, s in parts:
        z = R.restore(*[v.cpu().numpy() for v in L.kept[s]])
        (dxp, dxe), (dg, dge), dw = R.ffn_backward(x64, dy64, w, t, kk, g, z, a)
        np.add.at(want, t["perm"] // kk, dxp)
        np.add.at(bound, t["perm"] // kk, dxe + (kk + 3) * R.U32 * np.abs(dxp))
        if not s:
            within("dgate", L.dgate_w, dg.reshape(T, k), dge.reshape(T, k))
        for n in dw:
            within("grad " + s + n, L.grad[s + n], times * dw[n][0], times * dw[n][1] + (2 * times - 1) * 1.1 * R.U16 * np.abs(dw[n][0]) + 1e-30)
    within("dx", dx, want, bound + R.U16 * (np.abs(want) + bound))
    within("W_g", L.grad["W_g"], x64.T @ dl, (T + 2) * R.U32 * (np.abs(x64.T) @ np.abs(dl)))
    within("bias", L.grad["bias"], dl.sum(0), (T + 2) * R.U32 * np.abs(dl).sum(0))


def test_layer_after_an_optimizer_step():
    """pack(): what the forward products read follows the matrices."""
    torch, B, dev = _gpu()
    L, _ = trained_layer(70, 128, 192, 4, 2, "swiglu", 1, 64)
    M, _ = trained_layer(70, 128, 192, 4, 2, "swiglu", 1, 64, seed=2)
    x = torch.randn((70, 128), device=dev).bfloat16()
    want = M.forward(x).clone()
    for n, w in L.weight.items():
        w.copy_(M.weight[n])
    L.W_g.copy_(M.W_g)
    L.bias = M.bias
    L.pack()
    assert torch.equal(L.forward(x), want)


def test_layer_with_a_router_of_the_callers():
    torch, B, dev = _gpu()
    L, _ = trained_layer(70, 128, 192, 4, 2, "swiglu", 1)
    x, dy = torch.randn((70, 128), device=dev).bfloat16(), torch.randn((70, 128), device=dev)
    L.expert_idx.copy_(torch.stack([torch.randperm(4)[:2] for _ in range(70)]).int())
    L.gate_w.fill_(0.5)
    L.forward(x, routed=True)
    L.grad["W_g"].fill_(3.0)
    dx = L.backward(dy, x).double()
    assert (L.grad["W_g"] == 3).all()
    want = torch.zeros((70, 128), device=dev).index_add(0, L.perm.long() // 2, L.dx_perm)
    assert float((dx - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max()) * 1.01


def test_refused_calls_of_a_layer():
    torch, B, dev = _gpu()
    L, plain = trained_layer(9, 128, 64, 3, 1, "relu", 0)
    x, dy = torch.zeros((9, 128), dtype=torch.bfloat16, device=dev), torch.zeros((9, 128), device=dev)
    L.forward(x)
    for bad in ((dy[:8], x), (dy.double(), x), (dy, x.float()), (dy.cpu(), x), (dy.t().contiguous().t(), x)):
        with pytest.raises(B.MoeError):
            L.backward(*bad)
    with pytest.raises(B.MoeError):
        L.backward(dy, x, torch.zeros((9, 4), device=dev))
    with pytest.raises(B.MoeError):
        L.forward(x.float())
    with pytest.raises(AssertionError):
        plain.backward(dy, x)
    with pytest.raises(AssertionError):
        L.forward(x, rows=True)
    L.forward_few(x)                                       # (a decode step keeps nothing)
    with pytest.raises(AssertionError):
        L.backward(dy, x)
    L.expert_idx.fill_(0)
    L.forward(x, routed=True)
    with pytest.raises(AssertionError):
        L.backward(dy, x, torch.zeros((9, 3), device=dev))


@pytest.mark.parametrize("T,k,act,shared_F", [(48, 1, "relu", 0), (120, 2, "swiglu", 64)])
def test_block_for_inference_with_a_layer_that_trains(T, k, act, shared_F):
    torch, B, dev = _gpu()
    from paper_2506_12417_amd.block import MoEBlock
    L, _ = trained_layer(T, 256, 512, 4, k, act, 1 if k > 1 else 0, shared_F)
    h = torch.randn((T, 256), device=dev).bfloat16()
    out = []
    for train in (True, False):
        b = MoEBlock(L, pre="rms", next="rms", train=train)
        y, u = b.forward(h)
        out.append((y.clone(), u.clone()))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("T,k,act,shared_F", [(48, 1, "relu", 0), (120, 2, "swiglu", 64)])
def test_step_in_a_graph(T, k, act, shared_F):
    """A training step captured once and replayed with other inputs, with eager steps of another layer between: every replay gives the eager bits."""
    torch, B, dev = _gpu()
    from paper_2506_12417_amd.block import MoEBlock
    blocks = []
    for _ in range(2):
        L, _ = trained_layer(T, 256, 512, 4, k, act, 1 if k > 1 else 0, shared_F)
        b = MoEBlock(L, pre="rms", post="rms", next="layer", alpha=0.5, train=True)
        b.load(pre_w=np.full(256, 1.1, np.float32), next_w=np.full(256, 0.9, np.float32))
        blocks.append(b)
    h, dy, du = (torch.zeros((T, 256), dtype=torch.bfloat16, device=dev) for _ in range(3))

    def step(b, h, dy, du):
        b.forward(h)
        return b.backward(h, dy, du)[0]

    h.normal_(), dy.normal_(), du.normal_()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step(blocks[0], h, dy, du)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(blocks[0], h, dy, du)
    for i in range(4):
        h.normal_(), dy.normal_(), du.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = step(blocks[1], h, dy, du)
        assert torch.equal(out, want), i
        for a, b in ((blocks[0].grad, blocks[1].grad), (blocks[0].layer.grad, blocks[1].layer.grad)):
            assert all(a[n] is None or torch.equal(a[n], b[n]) for n in a), i


def test_block_backward_against_its_parts():
    torch, B, dev = _gpu()
    from paper_2506_12417_amd.block import MoEBlock
    T, d = 66, 192
    L, _ = trained_layer(T, d, 128, 5, 2, "swiglu", 1)
    b = MoEBlock(L, pre="layer", post="none", next="rms", alpha=1.0, train=True, h_dtype="f32")
    b.load(pre_w=np.ones(d, np.float32), pre_b=np.zeros(d, np.float32))
    h, dy, du = torch.randn((T, d), device=dev), torch.randn((T, d), device=dev), torch.randn((T, d), device=dev).bfloat16()
    b.forward(h)
    dh, none = b.backward(h, dy, du)
    assert none is None
    whole, grads = dh.clone(), {n: t.clone() for n, t in b.grad.items()}
    dv, _ = b.end_backward(h, dy, du)
    got = b.pre_backward(h, L.backward(dv, b.u))
    assert torch.equal(got, whole) and all(torch.equal(grads[n], b.grad[n]) for n in grads)
    # u made by the block before: its gradient comes back, and what the residual connection passes on
    u = b.u.clone()
    b.forward(h, u)
    dh, du_in = b.backward(h, dy, du)
    dv, dh2 = b.end_backward(h, dy, du)
    assert torch.equal(dh, dh2) and torch.equal(du_in, L.backward(dv, u))


def test_another_stream():
    torch, B, dev = _gpu()
    T, d, F, E, k, act = 130, 192, 128, 4, 2, "swiglu"
    (x, _), (dy, _), w, gate, rt = make_case(torch, T, d, F, E, k, act, {}, 4)
    q, scale = kept_values(torch, T * k, 2 * F, act, 1)
    w = {n: v[0] for n, v in w.items()}
    args = (torch, B, x, dy, w, torch.from_numpy(gate).to(dev), rt, torch.from_numpy(q).to(dev), torch.from_numpy(scale).to(dev), T, d, F, E, k, act)
    a = run_back(*args, dw_t=torch.bfloat16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = run_back(*args, dw_t=torch.bfloat16)
    s.synchronize()
    assert torch.equal(a[0][:T * k], b[0][:T * k]) and torch.equal(a[1], b[1]) and all(torch.equal(a[2][n], b[2][n]) for n in "abo")
