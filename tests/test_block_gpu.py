"""MoEBlock: pre norm, layer, gate, residual addition and the next block's norm, as a model runs them -- by one call for a few
tokens, with the combine folded into the end, or with it folded into the second product; two blocks behind one another; a training
step's backward calls.  The layer's own output is checked against the oracle elsewhere; here, what stands around it, and that the layer gets
what it should, bit for bit where the same sums are made."""
import numpy as np
import pytest

import moe_workloads as W
import test_norm_gpu as N
from gpu_util import make_layer

pytestmark = pytest.mark.gpu

NAMES = ("pre_w", "pre_b", "post_w", "post_b", "gate", "next_w", "next_b")


def make_block(T, d, F, E, k, dt, seed, shared_F=0, gate="none", post="none", next="rms", pre="rms", train=False, h_dtype="bf16", **kw):
    from paper_2506_12417_amd.block import MoEBlock
    wl = W.MoEWorkload("block", 6, T, d, F, E, k, "swiglu" if k > 1 else "relu", dt, 1, shared_F=shared_F)
    layer = make_layer(wl, W.make_inputs(wl, seed=seed))
    r = np.random.default_rng(seed)
    block = MoEBlock(layer, pre=pre, post=post, next=next, alpha=0.75, gate=gate, h_dtype=h_dtype, train=train, **kw)
    p = {n: 1.0 + 0.3 * r.standard_normal(d) if n.endswith("w") else 0.3 * r.standard_normal(d) for n in NAMES if n != "gate"}
    if gate != "none":
        p["gate"] = 0.5 + 0.3 * r.standard_normal(d if gate == "shared" else (T, d))
    block.load(**{n: a for n, a in p.items() if n in ("pre_w", "pre_b", "gate") or getattr(block, n.split("_")[0])})
    return block, r


def arguments(block, h, v):
    """What the formulas' reference takes."""
    np64 = lambda t: None if t is None else t.float().cpu().numpy().astype(np.float64)   # noqa: E731
    a = {n: np64(t) for n, t in block.param.items()}
    return dict(a, h=np64(h), v=None if v is None else np64(v), post=block.post, next=block.next, alpha=np.float32(block.alpha).item(), dy=None, du=None,
                gate=np64(block.param["gate"]) if block.gate_rows else None)


def check_pre(block, h):
    a = arguments(block, h, None)
    N.check("pre", block.u, N.reference(dict(a, v=None, gate=None, next=block.pre, next_w=a["pre_w"], next_b=a["pre_b"]))["u"], block.layer.dt)


@pytest.mark.parametrize("T,d,F,E,k,shared_F,dt", [(1, 768, 512, 8, 1, 0, "bf16"), (7, 320, 448, 12, 3, 64, "bf16"), (5, 320, 192, 6, 2, 0, "f32"),     # one call
                                                   (40, 512, 256, 9, 2, 128, "bf16"), (33, 192, 320, 5, 2, 64, "f32"), (300, 256, 192, 12, 4, 320, "bf16"),
                                                   (257, 768, 1024, 8, 1, 0, "bf16"), (900, 256, 512, 4, 1, 64, "bf16")])
@pytest.mark.parametrize("pre,post,next,gate,h_dtype", [("rms", "none", "rms", "none", "bf16"), ("layer", "rms", "layer", "token", "f32"),
                                                        ("rms", "layer", "none", "shared", "bf16")])
def test_block(T, d, F, E, k, shared_F, dt, pre, post, next, gate, h_dtype):
    torch, B = N._torch()
    print("[case] block", T, d, F, E, k, shared_F, dt, pre, post, next, gate, h_dtype, flush=True)
    from paper_2506_12417_amd.block import prefers_few
    block, r = make_block(T, d, F, E, k, dt, T + d, shared_F, gate, post, next, pre, h_dtype=h_dtype)
    L = block.layer
    h, _ = N.to_dev(torch, 2.0 * r.standard_normal((T, d)) + 0.2, block.h_dt)
    y, u_next = block.forward(h)
    torch.cuda.synchronize()
    assert prefers_few(L) == (T < 32) and y is block.y and (u_next is None) == (next == "none")
    check_pre(block, h)
    if not prefers_few(L):           # (the one call leaves v in the layer's buffer)
        L.forward(block.u)
    torch.cuda.synchronize()
    v = L.y.clone()
    if prefers_few(L):
        assert torch.equal(v, L.forward_few(block.u)) and not torch.isnan(v).any()
        close = (L.forward(block.u) - v).abs().max() / v.square().mean().sqrt()
        assert close <= (1e-5 if dt == "f32" else 1e-2), close          # (the general path's: other sums of the same)
    y2, u2 = torch.empty_like(y), None if u_next is None else torch.empty_like(u_next)
    p = block.param
    B.moe_block_end(v, B.MOE_F32, h, block.h_dt, T, d, block.post, block.eps, p["post_w"], p["post_b"], p["gate"], block.gate_rows, block.alpha, block.next,
                    block.eps, p["next_w"], p["next_b"], y2, u2, L.dt)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and (u_next is None or torch.equal(u_next, u2))
    ref = N.reference(arguments(block, h, v))
    N.check("y", y, ref["y"], block.h_dt)
    if u_next is not None:
        N.check("u", u_next, ref["u"], L.dt)


@pytest.mark.parametrize("T", [3, 200])
def test_two_blocks(T):
    """The second block takes the first one's u' in place of its own pre norm, on a stream of the caller's and in a graph."""
    torch, B = N._torch()
    (b1, r), (b2, _) = make_block(T, 512, 256, 8, 2, "bf16", 3, 128, "shared", "rms"), make_block(T, 512, 256, 8, 2, "bf16", 4)
    h, _ = N.to_dev(torch, r.standard_normal((T, 512)), B.MOE_BF16)

    def step():
        y, u = b1.forward(h)
        return b2.forward(y, u=u)

    y, u = step()
    torch.cuda.synchronize()
    want = y.clone(), u.clone(), b1.y.clone()
    v = b2.layer.forward_few(b1.u_next) if T == 3 else b2.layer.forward(b1.u_next)
    torch.cuda.synchronize()
    ref = N.reference(arguments(b2, want[2], v))
    N.check("y", want[0], ref["y"], B.MOE_BF16)
    N.check("u", want[1], ref["u"], B.MOE_BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(u, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        h.copy_(torch.randn(h.shape, generator=torch.Generator().manual_seed(seed)).to(h.dtype))
        step()
        torch.cuda.synchronize()
        want = y.clone(), u.clone()
        y.zero_()
        u.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(u, want[1])


@pytest.mark.parametrize("T,dt,h_dtype", [(9, "bf16", "bf16"), (130, "f32", "f32"), (333, "bf16", "f32")])
@pytest.mark.parametrize("post,next,gate", [("rms", "rms", "token"), ("layer", "none", "shared"), ("none", "layer", "none")])
def test_training_step(T, dt, h_dtype, post, next, gate):
    torch, B = N._torch()
    d = 192
    print("[case] block training", T, dt, h_dtype, post, next, gate, flush=True)
    block, r = make_block(T, d, 128, 6, 2, dt, T, 64, gate, post, next, "layer", train=True, h_dtype=h_dtype)
    h, _ = N.to_dev(torch, 2.0 * r.standard_normal((T, d)) + 0.2, block.h_dt)
    dy, _ = N.to_dev(torch, r.standard_normal((T, d)), block.h_dt)
    du, _ = N.to_dev(torch, r.standard_normal((T, d)), block.layer.dt)
    y, u = block.forward(h)
    dv, dh = block.end_backward(h, dy, du if block.next else None)
    torch.cuda.synchronize()
    a = dict(arguments(block, h, block.layer.y), dy=dy.float().cpu().numpy().astype(np.float64),
             du=du.float().cpu().numpy().astype(np.float64) if block.next else None)
    ref = N.reference(a)
    N.check("y", y, ref["y"], block.h_dt)
    N.check("dv", dv, ref["dv"])
    N.check("dh", dh, ref["dh"], block.h_dt)
    for n in ("dpost_w", "dpost_b", "dgate", "dnext_w", "dnext_b"):
        assert (n in block.grad) == (n in ref)
        if n in ref:
            N.check(n, block.grad[n], ref[n])
    # what the layer's backward would give for dv stands in: any gradient of u
    du_pre, _ = N.to_dev(torch, r.standard_normal((T, d)), block.layer.dt)
    a = arguments(block, h, None)
    ref = N.reference(dict(a, gate=None, next=block.pre, next_w=a["pre_w"], next_b=a["pre_b"], dy=dh.float().cpu().numpy().astype(np.float64),
                           du=du_pre.float().cpu().numpy().astype(np.float64)))
    dx = block.pre_backward(h, du_pre)
    torch.cuda.synchronize()
    N.check("dx", dx, ref["dh"], block.h_dt)
    N.check("dpre_w", block.grad["dpre_w"], ref["dnext_w"])
    N.check("dpre_b", block.grad["dpre_b"], ref["dnext_b"])


@pytest.mark.parametrize("T,post,next,gate", [(9, "rms", "rms", "token"), (130, "layer", "layer", "shared"), (40, "none", "rms", "none")])
def test_training_step_without_a_gradient_of_the_next_norms_output(T, post, next, gate):
    """du_next None is zero: all gradients as the formulas have them, those of the next norm's parameters zero."""
    torch, B = N._torch()
    print("[case] block training without du", T, post, next, gate, flush=True)
    block, r = make_block(T, 192, 128, 6, 2, "bf16", T, 64, gate, post, next, train=True)
    h, _ = N.to_dev(torch, 2.0 * r.standard_normal((T, 192)) + 0.2, block.h_dt)
    dy, _ = N.to_dev(torch, r.standard_normal((T, 192)), block.h_dt)
    block.forward(h)
    for g in block.grad.values():
        g.fill_(7.0)
    dv, dh = block.end_backward(h, dy, None)
    torch.cuda.synchronize()
    ref = N.reference(dict(arguments(block, h, block.layer.y), dy=dy.float().cpu().numpy().astype(np.float64)))
    N.check("dv", dv, ref["dv"])
    N.check("dh", dh, ref["dh"], block.h_dt)
    for n in ("dpost_w", "dpost_b", "dgate"):
        assert (n in block.grad) == (n in ref)
        if n in ref:
            N.check(n, block.grad[n], ref[n])
    assert not block.grad["dnext_w"].any() and not block.grad["dnext_b"].any()


@pytest.mark.parametrize("T,dt,h_dtype", [(9, "bf16", "bf16"), (333, "bf16", "f32"), (40, "f32", "f32")])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_two_trained_blocks(T, dt, h_dtype, norm):
    """The first block's next norm is the second one's pre norm, forward and backward: dh and the gradient of u go back to the first block's end.
    (Any gradients stand in for what the layers' own backward would give for dv.)"""
    torch, B = N._torch()
    d = 192
    print("[case] two trained blocks", T, dt, h_dtype, norm, flush=True)
    b1, r = make_block(T, d, 128, 6, 2, dt, T, 64, "shared", "rms", norm, train=True, h_dtype=h_dtype)
    b2, _ = make_block(T, d, 64, 4, 2, dt, T + 1, 0, "token", "layer", "rms", train=True, h_dtype=h_dtype)
    rows = lambda t: N.to_dev(torch, r.standard_normal((T, d)), t)[0]     # noqa: E731
    np64 = lambda t: t.float().cpu().numpy().astype(np.float64)   # noqa: E731
    h, dy2, du2, du_pre2, du_pre1 = rows(b1.h_dt), rows(b1.h_dt), *(rows(b1.layer.dt) for _ in range(3))
    y1, u1 = b1.forward(h)
    y2, u2 = b2.forward(y1, u=u1)
    dv2, dh2 = b2.end_backward(y1, dy2, du2)
    with pytest.raises(B.MoeError):
        b2.pre_backward(y1, du_pre2)
    dv1, dh1 = b1.end_backward(h, dh2, du_pre2)
    torch.cuda.synchronize()
    for b, into, dy, du, dv, dh in ((b2, y1, dy2, du2, dv2, dh2), (b1, h, dh2, du_pre2, dv1, dh1)):
        ref = N.reference(dict(arguments(b, into, b.layer.y), dy=np64(dy), du=np64(du)))
        N.check("y", b.y, ref["y"], b.h_dt)
        N.check("dv", dv, ref["dv"])
        N.check("dh", dh, ref["dh"], b.h_dt)
        for n in ("dpost_w", "dpost_b", "dgate", "dnext_w", "dnext_b"):
            N.check(n, b.grad[n], ref[n])
    # the second block took u as it was given, and the first one has a pre norm of its own
    v2 = b2.layer.y.clone()
    assert torch.equal(v2, b2.layer.forward_few(u1) if T == 9 else b2.layer.forward(u1))
    dh = dh1.clone()
    dx = b1.pre_backward(h, du_pre1)
    torch.cuda.synchronize()
    a = arguments(b1, h, None)
    ref = N.reference(dict(a, gate=None, next=b1.pre, next_w=a["pre_w"], next_b=a["pre_b"], dy=np64(dh), du=np64(du_pre1)))
    N.check("dx", dx, ref["dh"], b1.h_dt)
    N.check("dpre_w", b1.grad["dpre_w"], ref["dnext_w"])
    b2.forward(y1)                                    # (a forward of its own again: pre_backward is there)
    b2.pre_backward(y1, du_pre2)
    torch.cuda.synchronize()


@pytest.mark.parametrize("T,F,k,shared_F,dt", [(9, 128, 2, 64, "bf16"), (150, 128, 2, 64, "bf16"), (700, 512, 1, 0, "bf16"), (40, 128, 2, 0, "f32")])
def test_a_layer_runs_again_before_the_backward_calls(T, F, k, shared_F, dt):
    """The same layer in another trained block, and alone, by every form of its calls: the first block's gradients stay."""
    torch, B = N._torch()
    d = 256
    print("[case] tied layer", T, F, k, shared_F, dt, flush=True)
    b1, r = make_block(T, d, F, 6, k, dt, T, shared_F, "shared", "rms", "rms", train=True)
    from paper_2506_12417_amd.block import MoEBlock
    b2 = MoEBlock(b1.layer, post="rms", train=True)
    L = b1.layer
    rows = lambda t: N.to_dev(torch, r.standard_normal((T, d)), t)[0]     # noqa: E731
    h, other, dy, du = rows(b1.h_dt), rows(b1.h_dt), rows(b1.h_dt), rows(L.dt)
    b1.forward(h)
    want = [t.clone() for t in (*b1.end_backward(h, dy, du), *(b1.grad[n] for n in ("dpost_w", "dgate", "dnext_w")))]
    b1.forward(h)
    y = L.y.clone()
    b2.forward(other)
    x = rows(L.dt)
    alone = L.forward(x)
    assert alone is L.y and alone is not b1.v and alone is not b2.v
    if L.few_ok:
        assert L.forward_few(x) is alone
    got = [t.clone() for t in (*b1.end_backward(h, dy, du), *(b1.grad[n] for n in ("dpost_w", "dgate", "dnext_w")))]
    torch.cuda.synchronize()
    assert torch.equal(b1.v, y) and not torch.equal(b2.v, y) and not torch.equal(alone, y)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    mine = torch.full((T, d), float("nan"), device="cuda")
    assert L.forward(x, y=mine) is mine and L.y is mine
    got = mine.clone()
    torch.cuda.synchronize()
    assert torch.equal(got, L.forward(x))


def test_refusals():
    torch, B = N._torch()
    block, _ = make_block(5, 192, 128, 6, 2, "bf16", 1)
    with pytest.raises(AssertionError):
        block.load(pre_w=np.zeros(191))
    with pytest.raises(AssertionError):
        block.load(scale=np.zeros(192))
    with pytest.raises(AssertionError):
        block.load(gate=np.zeros(192))                 # (it has none)
    from paper_2506_12417_amd.block import MoEBlock
    gated = MoEBlock(block.layer, gate="shared")
    with pytest.raises(AssertionError):
        gated.forward(torch.zeros((5, 192), dtype=torch.bfloat16, device="cuda"))
    wide, _ = make_block(100, 192, 128, 6, 2, "bf16", 1)
    assert not wide.layer.few_ok
    with pytest.raises(AssertionError):
        wide.layer.forward_few(wide.u)
    fold, _ = make_block(257, 768, 1024, 8, 1, "bf16", 1)
    assert fold.layer.fold_combine
    with pytest.raises(AssertionError):
        fold.layer.forward(fold.u, rows=True)
