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
