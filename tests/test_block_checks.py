"""What MoEBlock and MoELayer.forward_few refuse before anything is enqueued (no GPU: the layer's buffers are in host memory)."""
import pytest
import torch

from paper_2506_12417_amd import binding as B
from paper_2506_12417_amd.block import MoEBlock, prefers_few
from paper_2506_12417_amd.layer import MoELayer

T, D = 6, 64


def block(dtype="bf16", h_dtype="f32", **kw):
    layer = MoELayer(T, D, 64, 4, 2, "relu", dtype, 0, device="cpu")
    layer.packed_router = dtype == "bf16"
    layer.W_gt = layer.w_norm2 = None
    return MoEBlock(layer, next="rms", h_dtype=h_dtype, **kw)


def refused(call, *args, status=B.MOE_ERR_ARG, **kw):
    with pytest.raises(B.MoeError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value


def bad_rows(dtype, other):
    """Tensors that are not T contiguous rows of D values of the type, and what they are refused with."""
    good = torch.zeros((T, D), dtype=dtype)
    return [(good.to(other), B.MOE_ERR_ARG), (good.double(), B.MOE_ERR_ARG), (good[:-1], B.MOE_ERR_ARG), (good[:, :-1], B.MOE_ERR_ARG),
            (torch.zeros((T + 1, D), dtype=dtype), B.MOE_ERR_ARG), (torch.zeros((D, T), dtype=dtype), B.MOE_ERR_ARG), (good.to("meta"), B.MOE_ERR_ARG),
            (good.numpy() if dtype == torch.float32 else [0.0], B.MOE_ERR_ARG), (torch.zeros((D, T), dtype=dtype).t(), B.MOE_ERR_UNSUPPORTED),
            (torch.zeros((T, 2 * D), dtype=dtype)[:, :D], B.MOE_ERR_UNSUPPORTED)]


def test_forward():
    b = block()
    h = torch.zeros((T, D))
    for t, status in bad_rows(torch.float32, torch.bfloat16):
        refused(b.forward, t, status=status)
    for t, status in bad_rows(torch.bfloat16, torch.float32):
        refused(b.forward, h, u=t, status=status)
        refused(b.layer.forward_few, t, status=status)
    x = torch.zeros((T, D), dtype=torch.bfloat16)
    for y in (torch.zeros((T, D), dtype=torch.float16), torch.zeros((T, D - 1)), torch.zeros((T, 2 * D))[:, :D]):
        refused(b.layer.forward_few, x, y=y, status=B.MOE_ERR_UNSUPPORTED if not y.is_contiguous() else B.MOE_ERR_ARG)


def test_backward():
    b = block(train=True)
    h, g, du = torch.zeros((T, D)), torch.zeros((T, D)), torch.zeros((T, D), dtype=torch.bfloat16)
    for t, status in bad_rows(torch.float32, torch.bfloat16):
        refused(b.end_backward, t, g, du, status=status)
        refused(b.end_backward, h, t, du, status=status)
        refused(b.pre_backward, t, du, status=status)
    for t, status in bad_rows(torch.bfloat16, torch.float32):
        refused(b.end_backward, h, g, t, status=status)
        refused(b.pre_backward, h, t, status=status)


def test_more_dimensions_and_one():
    """Rows of a batch of sequences, and values one behind the other, are the same memory: these pass on to the library (and fail for want of a
    GPU there)."""
    if torch.cuda.is_available():
        pytest.skip("for machines without a GPU: host addresses must not get there")
    b = block()
    for shape in ((2, 3, D), (T * D,), (T, D)):
        refused(b.forward, torch.zeros(shape), status=B.MOE_ERR_HIP)


def test_the_choice_follows_what_was_measured():
    """Sizes at which one form took at least 3 % longer than the other: that one is not chosen."""
    for few, sizes in ((True, ((1, 320, 512, 24, 4, "bf16"), (8, 320, 512, 24, 4, "bf16"), (8, 512, 512, 24, 4, "bf16"), (32, 768, 3072, 128, 1, "bf16"),
                               (24, 1024, 2048, 4, 1, "bf16"), (32, 2048, 2048, 8, 2, "bf16"), (32, 2048, 1408, 60, 4, "bf16"), (16, 1536, 768, 32, 4, "bf16"),
                               (16, 320, 1984, 16, 2, "f32"), (16, 1536, 1024, 6, 2, "f32"), (16, 1024, 2048, 8, 1, "f32"), (4, 1024, 2048, 8, 2, "f32"),
                               (6, 768, 1536, 16, 4, "f32"))),
                       (False, ((32, 320, 512, 24, 4, "bf16"), (32, 512, 512, 24, 4, "bf16"), (32, 768, 512, 16, 2, "bf16"), (24, 1088, 704, 24, 4, "bf16"),
                                (32, 1536, 768, 32, 4, "bf16"), (32, 512, 2048, 4, 2, "bf16"), (64, 4096, 14336, 8, 2, "bf16"), (64, 320, 512, 24, 4, "bf16"),
                                (12, 1024, 2048, 8, 2, "f32"), (16, 1024, 2048, 32, 2, "f32"), (8, 768, 1536, 16, 4, "f32"), (64, 320, 1984, 16, 2, "f32")))):
        for T, d, F, E, k, dtype in sizes:
            layer = MoELayer(T, d, F, E, k, "swiglu", dtype, 0, device="meta")
            layer.packed_router = dtype == "bf16"
            assert prefers_few(layer) == few, (T, d, F, E, k, dtype)
    layer = MoELayer(4, 320, 512, 8, 2, "swiglu", "bf16", 0, device="meta")
    assert not prefers_few(layer)                     # (its router is not packed)
