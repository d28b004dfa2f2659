"""A NaN in an expert's matrices through every family of the products' kernels: one in a first matrix makes the outputs of the tokens that
chose the expert NaN, one in a second matrix their outputs of that column, and all other values keep their bits.  (Not the fp32
products' ReLU: there the larger one of NaN and 0 is 0.)"""
import numpy as np
import pytest

import moe_workloads as W
from gpu_util import expert_dict, make_layer

pytestmark = pytest.mark.gpu

# mode: moe_ffn_kernel_mode (0 default, 1 LDS ring, 2 streaming); tile_m None: the library's choice
CASES = [(24, 192, 128, 6, 2, "relu", "bf16", 0, None), (24, 192, 128, 6, 2, "swiglu", "bf16", 0, None), (40, 256, 512, 4, 1, "relu", "bf16", 0, None),    # few rows
         (600, 512, 512, 4, 2, "relu", "bf16", 1, 128), (600, 512, 512, 4, 2, "swiglu", "bf16", 1, 128), (600, 512, 768, 4, 1, "relu", "bf16", 1, 128),    # LDS ring
         (600, 512, 512, 4, 2, "relu", "bf16", 2, 128), (600, 512, 512, 4, 2, "swiglu", "bf16", 2, 128),                                                  # streaming
         (900, 512, 512, 3, 2, "relu", "bf16", 0, 256), (900, 512, 512, 3, 2, "swiglu", "bf16", 0, 256), (900, 512, 512, 3, 1, "relu", "bf16", 0, 256),    # four wavefronts
         (20, 320, 192, 6, 2, "swiglu", "f32", 0, None), (700, 320, 448, 4, 2, "swiglu", "f32", 0, None)]                                                 # fp32


@pytest.mark.parametrize("T,d,F,E,k,act,dt,mode,tile_m", CASES)
def test_a_nan_in_a_matrix_reaches_the_outputs(T, d, F, E, k, act, dt, mode, tile_m):
    import torch
    from paper_2506_12417_amd import binding as B
    from paper_2506_12417_amd.layer import to_device
    assert torch.cuda.is_available(), "this test needs the MI355X"
    print("[case] NaN weights", T, d, F, E, k, act, dt, mode, tile_m, flush=True)
    before = B.moe_ffn_kernel_mode(-1)
    try:
        B.moe_ffn_kernel_mode(mode)
        wl = W.MoEWorkload("nan", 6, T, d, F, E, k, act, dt, 1)
        inp = W.make_inputs(wl, seed=T + F)
        layer = make_layer(wl, inp, tile_m=tile_m)
        x = to_device(inp["x"], layer.device)

        def run():
            layer.y.fill_(7.0)
            layer.forward(x)
            torch.cuda.synchronize()
            return layer.y.cpu().numpy().copy()

        y0, idx = run(), layer.expert_idx.cpu().numpy()
        assert np.isfinite(y0).all()
        e = int(np.bincount(idx.ravel(), minlength=E).argmax())
        chose = (idx == e).any(1)
        matrices = expert_dict(wl, inp)
        for name in matrices:
            w = {n: a[e].copy() for n, a in matrices.items()}
            w[name][w[name].shape[0] // 3, 17] = 0x7fc0 if dt == "bf16" else np.nan
            layer.experts.load_expert(e, w)
            y = run()
            want = np.zeros((T, d), dtype=bool)
            want[chose] = True
            if name in ("W2", "Wd"):
                want[:, :17] = want[:, 18:] = False
            assert np.array_equal(np.isnan(y), want) and np.array_equal(y[~want], y0[~want]), name
    finally:
        B.moe_ffn_kernel_mode(before)
