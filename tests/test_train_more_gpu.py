"""The training step beyond its single calls: what belongs to which pass of a layer, kernels that only large sizes take, extremes.  References in float64,
bounds as train_ref derives them."""
import numpy as np
import pytest

import train_ref as R
from test_train_gpu import _gpu, ints, rounded, run_back, trained_layer, within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ whose pass it is
def two_blocks(torch, T=70, d=128):
    from paper_2506_12417_amd.block import MoEBlock
    L, _ = trained_layer(T, d, 192, 4, 2, "swiglu", 1)
    blocks = [MoEBlock(L, pre="rms", next="rms", train=True) for _ in range(2)]
    h, dy, du = (torch.randn((T, d), device="cuda:0").bfloat16() for _ in range(3))
    return L, blocks, h, dy, du


def test_block_backward_refuses_another_pass_of_its_layer():
    torch, B, dev = _gpu()
    L, (a, b), h, dy, du = two_blocks(torch)
    a.forward(h)
    want = a.backward(h, dy, du)[0].clone()
    grads = {n: t.clone() for n, t in L.grad.items() if t is not None}
    between = {"another block": lambda: b.forward(-h), "an evaluation pass": lambda: L.forward(-h), "a decode step": lambda: L.forward_few(-h) if L.few_ok else L.route(-h),
               "the router": lambda: L.route(-h), "the sort": lambda: L.permute(None), "the sort and the plan": lambda: L.permute_plan()}
    for name, run in between.items():
        a.forward(h)
        run()
        dh = a.dh.fill_(3.0).clone()
        with pytest.raises(B.MoeError):
            a.backward(h, dy, du)
        assert torch.equal(a.dh, dh), name                 # (nothing has run)
    # the order that is right: a pass and its gradients, then the other block's; the same gradients again
    a.forward(h)
    assert torch.equal(a.backward(h, dy, du)[0], want) and torch.equal(a.backward(h, dy, du)[0], want)
    assert all(torch.equal(L.grad[n], g) for n, g in grads.items())
    b.forward(h)
    assert torch.equal(b.backward(h, dy, du)[0], want)
    # the gradients of all but the layer are the block's own, whatever the layer has done
    a.forward(h)
    dv = a.end_backward(h, dy, du)[0].clone()
    b.forward(-h)
    assert torch.equal(a.end_backward(h, dy, du)[0], dv)


def test_layer_backward_belongs_to_the_layers_last_pass():
    torch, B, dev = _gpu()
    L, _, h, dy, _ = two_blocks(torch)
    for run in (lambda: L.route(h), lambda: L.permute(None), lambda: L.permute_plan()):
        L.forward(h)
        L.backward(dy, h)
        run()
        with pytest.raises(AssertionError):
            L.backward(dy, h)
    # a pass that was refused keeps nothing
    L.forward(h)

    def refused(stream=None):
        raise B.MoeError(B.MOE_ERR_ARG, "refused")

    L.permute_plan = refused
    with pytest.raises(B.MoeError):
        L.forward(h)
    del L.permute_plan
    with pytest.raises(AssertionError):
        L.backward(dy, h)


def test_block_that_is_not_trained_has_no_backward():
    torch, B, dev = _gpu()
    from paper_2506_12417_amd.block import MoEBlock
    L, (a, _), h, dy, du = two_blocks(torch)
    plain = MoEBlock(L, pre="rms", next="rms")
    plain.forward(h)
    with pytest.raises(B.MoeError):
        plain.backward(h, dy, du)
    with pytest.raises(B.MoeError):
        a.backward(h, dy, du)                              # (its own forward() has not run)


# ------------------------------------------------------------------------------------------------ in place
@pytest.mark.parametrize("T,d,k", [(1, 5000, 1), (1, 4096, 1), (77, 777, 3), (130, 2048, 4), (3, 8, 9), (2000, 513, 2)])
def test_permute_backward_adds_in_place(T, d, k):
    torch, B, dev = _gpu()
    rows, add, inv = torch.randn((T * k, d), device=dev), torch.randn((T, d), device=dev), torch.randperm(T * k, device=dev).int()
    dx = torch.empty((T, d), device=dev)
    B.moe_permute_backward(rows, inv, T, d, k, add, dx, B.MOE_F32)
    want = add.double() + rows.double()[inv.long()].reshape(T, k, d).sum(1)
    mag = add.double().abs() + rows.double().abs()[inv.long()].reshape(T, k, d).sum(1)
    assert ((dx.double() - want).abs() <= (k + 1) * R.U32 * mag).all()
    B.moe_permute_backward(rows, inv, T, d, k, add, add, B.MOE_F32)
    assert torch.equal(dx, add)


# ------------------------------------------------------------------------------------------------ micro-batches
def check_sums(torch, names, got, one, two):
    """fp32 gradients are added with one rounding, bf16 ones are rounded once a call."""
    assert names
    for n in names:
        a, b, s = one[n].double(), two[n].double(), got[n].double()
        if got[n].dtype == torch.float32:
            assert torch.equal(got[n], one[n] + two[n]), n
        else:
            assert ((s - a - b).abs() <= R.U16 * 1.01 * (b.abs() + s.abs())).all(), n


@pytest.mark.parametrize("gate,post,next_,pre,du_next,shared_F", [("none", "rms", "rms", "rms", True, 64), ("shared", "layer", "layer", "layer", True, 0),
                                                                  ("token", "none", "rms", "layer", False, 0)])
def test_block_adds_up_all_gradients(gate, post, next_, pre, du_next, shared_F):
    torch, B, dev = _gpu()
    from paper_2506_12417_amd.block import MoEBlock
    T, d = 70, 128
    r = np.random.default_rng(5)
    par = {n: r.standard_normal(d).astype(np.float32) for n in ("pre_w", "post_w", "next_w")}
    par.update({n: r.standard_normal(d).astype(np.float32) for n, kind in (("pre_b", pre), ("post_b", post), ("next_b", next_)) if kind == "layer"})
    if post == "none":
        del par["post_w"]
    if gate != "none":
        par["gate"] = r.standard_normal((1 if gate == "shared" else T, d)).astype(np.float32)

    def made():
        L, _ = trained_layer(T, d, 192, 4, 2, "swiglu", 1, shared_F)
        b = MoEBlock(L, pre=pre, post=post, next=next_, gate=gate, alpha=0.5, train=True)
        b.load(**par)
        return b

    def grads(b):
        return {n: t.clone() for n, t in list(b.grad.items()) + [("layer " + n, t) for n, t in b.layer.grad.items() if t is not None]}

    batches = [[torch.randn((T, d), device=dev).bfloat16() for _ in range(3)] for _ in range(2)]
    alone = []
    for h, dy, du in batches:
        b = made()
        b.forward(h)
        dh = b.backward(h, dy, du if du_next else None)[0]
        alone.append((grads(b), dh.clone()))
    b = made()
    for i, (h, dy, du) in enumerate(batches):
        b.forward(h)
        dh = b.backward(h, dy, du if du_next else None, accumulate=i > 0)[0]
        assert torch.equal(dh, alone[i][1])
    assert set(b.grad) == {"d" + n for n in par}
    check_sums(torch, list(alone[0][0]), grads(b), alone[0][0], alone[1][0])
    # without it everything is set again
    b.forward(batches[0][0])
    b.backward(*batches[0][:2], batches[0][2] if du_next else None)
    assert all(torch.equal(alone[0][0][n], t) for n, t in grads(b).items())


def test_block_adds_up_where_u_is_given_and_in_a_graph():
    torch, B, dev = _gpu()
    from paper_2506_12417_amd.block import MoEBlock
    T, d = 48, 256
    L, _ = trained_layer(T, d, 512, 4, 1, "relu", 0)
    b = MoEBlock(L, pre="rms", next="rms", train=True)
    b.load(pre_w=np.full(d, 1.1, np.float32), next_w=np.full(d, 0.9, np.float32))
    h, u, dy, du = (torch.randn((T, d), device=dev).bfloat16() for _ in range(4))
    b.forward(h, u)
    b.backward(h, dy, du)
    one, pre = {n: t.clone() for n, t in L.grad.items() if t is not None}, b.grad["dpre_w"].fill_(3.0).clone()
    b.forward(h, u)
    b.backward(h, dy, du, accumulate=True)
    assert torch.equal(b.grad["dpre_w"], pre)              # (the pre norm has not run: its gradients are another block's)
    assert torch.equal(L.grad["W_g"], 2 * one["W_g"]) and torch.equal(L.grad["bias"], 2 * one["bias"])
    b.forward(h)
    b.backward(h, dy, du)
    first = {n: t.clone() for n, t in list(b.grad.items()) + [("layer " + n, t) for n, t in L.grad.items() if t is not None]}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward(h)
        b.backward(h, dy, du, accumulate=True)
    for i in range(3):
        for n, t in list(b.grad.items()) + [("layer " + n, t) for n, t in L.grad.items() if t is not None]:
            t.copy_(first[n])
        graph.replay()
        torch.cuda.synchronize()
        for n in ("dpre_w", "dnext_w", "layer W_g", "layer bias"):
            assert torch.equal((L.grad[n[6:]] if n.startswith("layer") else b.grad[n]), 2 * first[n]), (i, n)


def test_layer_adds_up_the_routers_gradients_too():
    torch, B, dev = _gpu()
    L, _ = trained_layer(70, 128, 192, 4, 2, "swiglu", 1)
    M, _ = trained_layer(70, 128, 192, 4, 2, "swiglu", 1)
    xs, dys, extra = [torch.randn((70, 128), device=dev).bfloat16() for _ in range(2)], [torch.randn((70, 128), device=dev) for _ in range(2)], torch.randn((70, 4), device=dev)
    alone = []
    for x, dy in zip(xs, dys):
        M.forward(x)
        M.backward(dy, x, extra)
        alone.append({n: t.clone() for n, t in M.grad.items() if t is not None})
    for i in range(2):
        L.forward(xs[i])
        L.backward(dys[i], xs[i], extra, accumulate=i > 0, accumulate_router=i > 0)
    check_sums(torch, list(alone[0]), L.grad, *alone)
    # the choice was the caller's: the router's gradients are left alone
    held = {n: L.grad[n].clone() for n in ("W_g", "bias")}
    L.forward(xs[0], routed=True)
    L.backward(dys[0], xs[0], accumulate=True, accumulate_router=True)
    assert all(torch.equal(L.grad[n], t) for n, t in held.items())


# ------------------------------------------------------------------------------------------------ extremes
@pytest.mark.parametrize("act", ["relu", "swiglu"])
def test_scales_at_the_end_of_fp32(act):
    """q scale is a number where 128 scale is not."""
    torch, B, dev = _gpu()
    from test_train_gpu import make_case
    T, d, F, E, k = 75, 128, 192, 3, 2
    (x, x64), (dy, dy64), w, gate, rt = make_case(torch, T, d, F, E, k, act, {}, 6)
    r = np.random.default_rng(7)
    A, big = T * k, np.float32(2.67e36)
    assert 128 * float(big) > float(np.finfo(np.float32).max) > 127 * float(big)
    q = r.integers(0, 128, (A, F))
    q[r.random((A, F)) < 0.2] = 0
    scale = np.full((A, F // 64), big)
    if act == "swiglu":                                    # (gates at or below zero: silu is 0 there; ups of any size)
        q = np.concatenate([-q, r.integers(-127, 128, (A, F))], 1)
        scale = np.concatenate([scale, (r.random((A, F // 64)) * 0.04).astype(np.float32)], 1)
    q = q.astype(np.int8)
    w32, w64 = {n: v[0] for n, v in w.items()}, {n: v[1] for n, v in w.items()}
    dx, dgate, dw = run_back(torch, B, x, dy, w32, torch.from_numpy(gate).to(dev), rt, torch.from_numpy(q).to(dev), torch.from_numpy(scale).to(dev), T, d, F, E, k, act,
                             dw={n: None for n in "abo"} if act == "relu" else None, dw_t=torch.float32, dgate=act == "swiglu")
    with np.errstate(over="ignore"):
        (dxp, dxe), (dg, dge), ref = R.ffn_backward(x64, dy64, w64, rt, k, gate.astype(np.float64), R.restore(q, scale), act)
    within("dx_perm", dx[:A], dxp, dxe)
    if act == "swiglu":
        within("dgate_w", dgate, dg.reshape(T, k), dge.reshape(T, k))
        for n in ref:
            within("dw " + n, dw[n], ref[n][0], ref[n][1] + np.abs(ref[n][0]) * R.U32)


# ------------------------------------------------------------------------------------------------ sums that are exact
# Whole numbers (times powers of two) of few bits: every product and sum below is a number that its type holds, so that the gradients have to be equal to
# the definition's to the last bit, and a row that is missing, doubled or of another place shows.  dy, x and the matrices hold -1, 0 and 1, gates and hidden
# values powers of two; SwiGLU's gates are 32, 64 and 128, whose sigmoid is 1 in fp32.  s is a sum of d such terms: below 256 it has bf16's 8 bits.
BIG = [  # T, d, F, E, k, act, rows of the experts by weight (0: none)
    (33000, 1088, 64, 4, 1, "relu", (3, 0, 5, 1)),         # (256 rows a tile for dx)
    (33000, 1088, 64, 4, 1, "swiglu", (3, 0, 5, 1)),       # (and the second matrix behind the first)
    (16500, 2112, 1088, 4, 2, "swiglu", (4, 3, 2, 1)),     # (and tiles of 256 x 256 for dW)
    (2400, 576, 832, 24, 2, "relu", None),
    (2400, 576, 832, 24, 2, "swiglu", None),               # (tiles of 256 x 256, some hundred ragged rows an expert, two panels' remainders)
    (1300, 320, 2112, 40, 1, "relu", None),
    (700, 192, 448, 5, 3, "swiglu", None),                 # (tiles of 128 x 128)
    (98304, 64, 14336, 2, 1, "swiglu", (1, 900)),          # (offsets beyond 2^32 bytes)
]


def whole_case(torch, T, d, F, E, k, act, weights, seed):
    dev, gen = "cuda:0", torch.Generator(device="cuda:0").manual_seed(seed)
    three = lambda *shape: torch.randint(-1, 2, shape, device=dev, generator=gen).bfloat16()      # noqa: E731
    p = torch.tensor(weights if weights else [1.0 + e % 4 for e in range(E)], device=dev, dtype=torch.float32)
    idx = torch.multinomial(p.expand(T, E), k, generator=gen)
    flat = idx.reshape(-1)
    perm = torch.sort(flat, stable=True)[1]
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(T * k, device=dev)
    counts = torch.bincount(flat, minlength=E).tolist()
    rt = dict(offsets=np.concatenate([[0], np.cumsum(counts)]), perm=perm.cpu().numpy(), inv=inv.cpu().numpy(), counts=counts)
    w = {n: three(E, d, F) for n in ("ab" if act == "swiglu" else "a")}
    w["o"] = three(E, F, d)
    gate = 2.0 ** torch.randint(-1, 2, (T, k), device=dev, generator=gen).float()
    A, nb = T * k, F // 64
    if act == "relu":
        q = torch.randint(-3, 3, (A, F), device=dev, generator=gen, dtype=torch.int8)
        q = torch.where(q < 0, 0, 2 ** q.clamp_min(0)).to(torch.int8)
        scale = 2.0 ** torch.randint(-1, 2, (A, nb), device=dev, generator=gen).float()
    else:
        q = torch.empty((A, 2 * F), dtype=torch.int8, device=dev)
        q[:, :F] = 32 * 2 ** torch.randint(0, 2, (A, F), device=dev, generator=gen, dtype=torch.int8)
        q[:, F:] = torch.randint(-2, 3, (A, F), device=dev, generator=gen, dtype=torch.int8)
        scale = 2.0 ** torch.randint(0, 2, (A, 2 * nb), device=dev, generator=gen).float()
    return three(T, d), three(T, d), w, gate, rt, q, scale


def check_whole(torch, got, x, dy, w, gate, rt, q, scale, T, d, F, E, k, act, before=None):
    dx_perm, dgate_w, dw = got
    dgate = torch.zeros(T * k, dtype=torch.float64, device="cuda:0")
    for e in range(E):
        sl = slice(int(rt["offsets"][e]), int(rt["offsets"][e + 1]))
        a = torch.from_numpy(rt["perm"][sl]).to("cuda:0")
        X, DY, g = x[a // k].double(), dy[a // k].double(), gate.reshape(-1)[a].double()[:, None]
        dx = torch.zeros((len(a), d), dtype=torch.float64, device="cuda:0")
        for f in range(0, F, 1088):
            cols = slice(f, min(f + 1088, F))
            kept = [q[sl, m * F + f:m * F + cols.stop].double() * scale[sl].double().repeat_interleave(64, 1)[:, m * F + f:m * F + cols.stop] for m in range(len(w) - 1)]
            s = DY @ w["o"][e][cols].double().t()
            assert float(s.abs().max() if len(a) else 0) < 256
            if act == "relu":
                h, dz = kept[0], [g * s * (kept[0] > 0)]
            else:
                h, dz = kept[0] * kept[1], [g * s * kept[1], g * s * kept[0]]
            dgate[a] += (h * s).sum(1)
            want = {"o": (g * h).t() @ DY}
            for n, v in zip("ab", dz):
                want[n] = X.t() @ v
                dx += v @ w[n][e][:, cols].double().t()
            for n, v in want.items():
                out = dw[n][e][cols] if n == "o" else dw[n][e][:, cols]
                if before is not None:
                    v = v + (before[n][e][cols] if n == "o" else before[n][e][:, cols]).double()
                assert float(v.abs().max()) < 2 ** 24 and torch.equal(out, v.to(out.dtype)), (e, n, f)
        if dx_perm is not None:
            assert torch.equal(dx_perm[sl], dx.float()), e
    if dgate_w is not None:
        assert torch.equal(dgate_w.reshape(-1), dgate.float())


@pytest.mark.parametrize("T,d,F,E,k,act,weights", BIG)
def test_gradients_of_whole_numbers(T, d, F, E, k, act, weights):
    torch, B, dev = _gpu()
    print("[case] whole numbers", T, d, F, E, k, act, flush=True)
    x, dy, w, gate, rt, q, scale = case = whole_case(torch, T, d, F, E, k, act, weights, T + d)
    args = (torch, B, x, dy, w, gate, rt, q, scale, T, d, F, E, k, act)
    for t in (torch.bfloat16, torch.float32):
        got = run_back(*args, dw_t=t)
        check_whole(torch, got, *case, T, d, F, E, k, act)
        if T > 50000:
            return
        before = {n: v.clone() for n, v in got[2].items() if v is not None}
        _, _, dw = run_back(*args, dw=got[2], accumulate=1, dgate=False, dxp=False)
        check_whole(torch, (None, None, dw), *case, T, d, F, E, k, act, before=before)


def test_whole_numbers_show_a_lost_row():
    """The check itself, with an oracle that lacks a row's share, and one that has another row's."""
    torch, B, dev = _gpu()
    T, d, F, E, k, act, weights = BIG[6]
    x, dy, w, gate, rt, q, scale = whole_case(torch, T, d, F, E, k, act, weights, 1)
    got = run_back(torch, B, x, dy, w, gate, rt, q, scale, T, d, F, E, k, act, dw_t=torch.float32)
    check_whole(torch, got, x, dy, w, gate, rt, q, scale, T, d, F, E, k, act)
    for other in (torch.cat([x[:-1], torch.zeros_like(x[:1])]), x.flip(0)):
        with pytest.raises(AssertionError):
            check_whole(torch, got, other, dy, w, gate, rt, q, scale, T, d, F, E, k, act)


@pytest.mark.parametrize("T,d,F,E,k,act,renorm,shared_F", [(2600, 256, 512, 4, 1, "relu", 0, 0), (1900, 320, 192, 3, 2, "swiglu", 1, 128)])
def test_layer_of_many_rows_an_expert(T, d, F, E, k, act, renorm, shared_F):
    """The second product on tall tiles, of what the first one has left."""
    import test_train_gpu
    test_train_gpu.test_layer(T, d, F, E, k, act, renorm, shared_F)
