"""A MoE layer as it stands in a model, between two residual additions:

    u = pre(h),   v = layer(u),   y = alpha * h + gate * post(v),   u' = next(y)

Like the layer, this owns buffers and marshals arguments; every value is computed in the library's kernels."""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import numpy as np
import torch

from . import binding as B
from .layer import MoELayer, to_device

KINDS = {"none": B.MOE_NORM_NONE, "rms": B.MOE_NORM_RMS, "layer": B.MOE_NORM_LAYER}
NAMES = ("pre_w", "pre_b", "post_w", "post_b", "gate", "next_w", "next_b")


def prefers_few(layer: MoELayer) -> bool:
    """Whether one call serves the layer's tokens better than the separate ones.  Measured: a block with the next norm, us by this call / by
    those, in graphs over enough layers that no weight is in a cache.

    16 bits, up to 16 tokens: d=768 F=3072 E=128 k=1 one token 27 / 32, 16 tokens 48 / 55; d=2048 F=1408 E=60 k=4 with a shared expert 8 tokens 103 / 119;
    d=320 F=512 E=24 k=4 16 tokens 31 / 32, d=960 F=1472 E=8 k=2 41 / 39.  Up to 32 where they choose one expert each or d is beyond 1536: d=768 F=3072
    62 / 71, d=1024 F=2048 E=4 k=1 28 / 32, d=2048 F=2048 E=8 k=2 52 / 58, d=2048 F=1408 164 / 177.  Not in narrower layers, where an expert's matrices
    are fetched, or its rows multiplied, once for every range of tokens: d=512 F=512 E=24 k=4 39 / 36, d=512 F=2048 E=4 k=2 38 / 33, d=1536 F=768
    E=32 k=4 72 / 69.  Beyond, whole tiles of rows are worth a plan.

    fp32, up to 16 tokens: d=320 F=1984 E=16 k=2 5 tokens 30 / 35, 16 tokens 38 / 40; d=1536 F=1024 E=6 k=2 16 tokens 39 / 42.  The matrix instruction
    bounds both, and where ranges of tokens share the columns (d up to 1024, more choices than one) 2^25 multiply-adds a matrix, all rows counted, are
    the line: d=768 F=1536 E=16 k=4 6 tokens 51 / 53, 8 tokens 58 / 54; d=1024 F=2048 E=8 k=2 4 tokens 40 / 46, 8 tokens 50 / 50, 12 tokens 58 / 51."""
    T, d, k = layer.T, layer.d, layer.k
    if not layer.few_ok:
        return False
    if layer.dt == B.MOE_BF16:
        return layer.packed_router and T <= (32 if k == 1 or d > 1536 else 16)
    return T <= 16 and (k == 1 or d > 1024 or T * k * d * layer.F < 2 ** 25)


class MoEBlock:
    """pre, post, next: "rms", "layer" or "none" (pre always is one; next is the norm of the block behind, whose u' comes out here).
    h_dtype: the residual stream's type; the layer's own is u's.  gate: "none", "shared" (one row of d factors) or "token" (a row for every
    token).  train: forward() keeps what the backward calls read, and v is stored for them."""

    def __init__(self, layer: MoELayer, pre: str = "rms", post: str = "none", next: str = "none", eps: float = 1e-5, alpha: float = 1.0,
                 gate: str = "none", h_dtype: str = "bf16", train: bool = False):
        assert pre != "none" and layer.d <= B.MOE_NORM_MAX_D
        self.layer, self.eps, self.alpha, self.train = layer, eps, alpha, train
        self.T, self.d, dev = layer.T, layer.d, layer.device
        self.pre, self.post, self.next = KINDS[pre], KINDS[post], KINDS[next]
        self.gate_rows = {"none": 0, "shared": 1, "token": self.T}[gate]
        self.h_dt = B.MOE_BF16 if h_dtype == "bf16" else B.MOE_F32
        self.h_tdt = torch.bfloat16 if h_dtype == "bf16" else torch.float32
        self.param: Dict[str, Optional[torch.Tensor]] = {n: None for n in NAMES}
        T, d, f32 = self.T, self.d, torch.float32
        self.u = torch.empty((T, d), dtype=layer.tdt, device=dev)
        self.y = torch.empty((T, d), dtype=self.h_tdt, device=dev)
        self.u_next = torch.empty((T, d), dtype=layer.tdt, device=dev) if self.next else None
        # (trained, the block keeps v itself: the layer may run again, for another block or alone, before the backward calls)
        self.v = torch.empty((T, d), dtype=f32, device=dev) if train else None
        if train:
            self.pre_stats = torch.empty((T, 2), dtype=f32, device=dev)
            self.end_stats = torch.empty((T, 4), dtype=f32, device=dev)
            self.grad: Dict[str, torch.Tensor] = {}
            n = max(B.moe_workspace_bytes(op, T, d, 0, 0, 0, layer.dt) for op in (B.MOE_OP_NORM_BACKWARD, B.MOE_OP_BLOCK_END_BACKWARD))
            self.ws = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
            self.dv = torch.empty((T, d), dtype=f32, device=dev)
            self.dh = torch.empty((T, d), dtype=self.h_tdt, device=dev)
            self.pre_own = True              # whether the last forward() has run the pre norm

    def load(self, **arrays: np.ndarray):
        """Parameters by name (NAMES), fp32: [d], and the gate [d] or [T,d].  What is not loaded counts as ones (weights) or zeros."""
        for name, a in arrays.items():
            rows = self.gate_rows if name == "gate" else 1
            assert name in NAMES and rows and np.shape(a) in (((self.d,), (1, self.d)) if rows == 1 else ((rows, self.d),)), name
            self.param[name] = to_device(np.asarray(a, dtype=np.float32).reshape(-1, self.d), self.layer.device)
            if self.train:
                self.grad["d" + name] = torch.empty_like(self.param[name])

    def _check(self, dtype: torch.dtype, **tensors: Optional[torch.Tensor]):
        for name, t in tensors.items():
            if t is not None:
                B.check_rows(name, t, self.T, self.d, (dtype,), self.y.device)

    def _end(self) -> Tuple:
        p = self.param
        assert self.gate_rows == 0 or p["gate"] is not None, "the gate is not loaded"
        return (self.T, self.d, self.post, self.eps, p["post_w"], p["post_b"], p["gate"] if self.gate_rows else None, self.gate_rows, self.alpha,
                self.next, self.eps, p["next_w"], p["next_b"], self.y, self.u_next, self.layer.dt)

    def forward(self, h: torch.Tensor, u: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """Enqueues the block; returns y and u' (None without a next norm), buffers of the block's own.  u: pre(h), where the block before has
        made it as its u' (its next norm stands in for this one's pre norm, and so it is in the backward calls: the gradient of u goes to that
        block's end_backward as du_next, this one's dh as dy, and there is no pre_backward)."""
        L, p = self.layer, self.param
        self._check(self.h_tdt, h=h)
        self._check(L.tdt, u=u)
        self.pre_own = u is None
        if u is None:
            B.moe_norm(h, self.h_dt, p["pre_w"], p["pre_b"], self.T, self.d, self.pre, self.eps, self.u, L.dt, self.pre_stats if self.train else None,
                       stream)
            u = self.u
        if prefers_few(L):
            L.forward_few(u, self.v, stream)
        elif self.train or L.fold_combine:
            L.forward(u, stream, y=self.v)
        else:
            # the layer's combine in the same pass as what follows it: v is never stored
            L.forward(u, stream=stream, rows=True)
            B.moe_block_end_rows(L.y_perm, L.inv_perm, L.gate_w, L.s_y if L.shared_F else None, L.k, h, self.h_dt, *self._end(), stream)
            return self.y, self.u_next
        B.moe_block_end(L.y, B.MOE_F32, h, self.h_dt, *self._end(), self.end_stats if self.train else None, stream)
        return self.y, self.u_next

    def end_backward(self, h: torch.Tensor, dy: Optional[torch.Tensor], du_next: Optional[torch.Tensor], stream=None):
        """From the gradients of y and u' to those of v (fp32) and, by the residual connection, of h; the parameters' go to `grad`.  Either of dy
        and du_next may be None, which is zero: without du_next the gradients of the next norm's parameters are."""
        p, g = self.param, self.grad
        self._check(self.h_tdt, h=h, dy=dy)
        self._check(self.layer.tdt, du_next=du_next)
        of_next = g.get("dnext_w"), g.get("dnext_b")
        B.moe_block_end_backward(dy, du_next, self.layer.dt, self.v, B.MOE_F32, h, self.h_dt, self.T, self.d, self.post, p["post_w"], p["post_b"],
                                 p["gate"] if self.gate_rows else None, self.gate_rows, self.alpha, self.next, p["next_w"], self.end_stats, self.dv, self.dh,
                                 *[g.get(n) for n in ("dpost_w", "dpost_b", "dgate")], *((None, None) if du_next is None else of_next), self.ws, self.ws.numel(), stream)
        if du_next is None and of_next != (None, None):
            # (gradients over no tokens: zero)
            B.moe_norm_backward(None, self.layer.dt, None, self.h_dt, None, None, 0, self.d, self.next, None, None, *of_next, None, 0, stream)
        return self.dv, self.dh

    def pre_backward(self, h: torch.Tensor, du: torch.Tensor, stream=None) -> torch.Tensor:
        """From the gradient of u, as the layer's own backward gives it for dv, to h's whole gradient: end_backward's dh is added, in
        place."""
        p, g = self.param, self.grad
        if not self.pre_own:
            raise B.MoeError(B.MOE_ERR_ARG, "forward() was given u: its gradient is du_next of the block that has made it")
        self._check(self.h_tdt, h=h)
        self._check(self.layer.tdt, du=du)
        B.moe_norm_backward(du, self.layer.dt, h, self.h_dt, p["pre_w"], self.pre_stats, self.T, self.d, self.pre, self.dh, self.dh, g.get("dpre_w"),
                            g.get("dpre_b"), self.ws, self.ws.numel(), stream)
        return self.dh
