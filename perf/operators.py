"""Performance cases of the operators around the MoE layer: the norms before and after a block, with its gate
and residual scale, forward and backward, and a whole MoE layer for a few tokens.

Kinds of case:

  few       one MoE layer for at most 64 tokens (a decode step): routing, experts, combine
  norm      the norm before a block; with train, its gradients too
  end       the end of a block: norm of its output, gate, residual scale, the next block's norm; with train, its gradients too
  end_rows  the same where the block's output is still the experts' rows, to be weighted and summed

All inputs are drawn on the GPU from the seed alone: activations and gradients N(0,1), matrices N(0,1/fan_in), a router bias that gives
the experts roughly Zipf-distributed loads, norm weights around one.  Plain form: elementary torch operations in 32 bits.
"""
import math

import torch

own = False
DEV = "cuda:0"
NORMS = {"none": 0, "rms": 1, "layer": 2}


# ------------------------------------------------------------------------------------- the cases
def listed():
    switch = dict(kind="few", d=768, F=3072, E=128, k=1, act="relu", dtype="bf16", renorm=0, shared_F=0, zipf=1.0)
    return [
        # one sequence's decode step through the smallest experts: launches and latencies
        dict(switch, name="few_one_token", T=1),
        # eight sequences, one token each, top-1 routing over many experts
        dict(switch, name="few_switch", T=8),
        # fine-grained experts and a shared one, as many sequences as make nearly all experts active
        dict(name="few_fine", kind="few", T=33, d=2048, F=1408, E=60, k=4, act="swiglu", dtype="bf16", renorm=0, shared_F=5632, zipf=1.2),
        # large experts, a handful of sequences: the fetch of the chosen experts' weights is the work
        dict(name="few_large", kind="few", T=3, d=4096, F=14336, E=8, k=2, act="swiglu", dtype="bf16", renorm=1, shared_F=0, zipf=1.0),
        # a layer kept in fp32
        dict(name="few_f32", kind="few", T=5, d=320, F=1984, E=16, k=2, act="swiglu", dtype="f32", renorm=1, shared_F=0, zipf=1.0),
        # the norm of a decode step
        dict(name="norm_decode", kind="norm", T=8, d=4096, norm="rms", bias=False, dtype="bf16", train=False),
        # a training step's norm before the layer, at the benchmark's sizes
        dict(name="norm_train", kind="norm", T=16384, d=2048, norm="layer", bias=True, dtype="bf16", train=True),
        # fp32, a width that is no multiple of anything
        dict(name="norm_f32_odd", kind="norm", T=1501, d=777, norm="rms", bias=False, dtype="f32", train=True),
        # the end of a block in a decode step, with the next block's norm
        dict(name="end_decode", kind="end", T=33, d=2048, post="rms", gate="channel", alpha=1.0, next="rms", bias=False, dtype="bf16", train=False),
        # the layer's own end at prefill: four rows a token and a shared expert's output, residual, next norm
        dict(name="end_rows_prefill", kind="end_rows", T=8192, d=2048, k=4, shared=True, post="none", gate="none", alpha=1.0, next="rms",
             bias=False, dtype="bf16", train=False),
        # training with norms on both sides, a learned gate per channel and a scaled residual
        dict(name="end_train", kind="end", T=8192, d=4096, post="rms", gate="channel", alpha=0.81, next="rms", bias=False, dtype="bf16", train=True),
        # a gate of every token's own (made by a small network), biases, a ragged width, fp32
        dict(name="end_token_gate", kind="end", T=1501, d=1032, post="layer", gate="token", alpha=1.0, next="layer", bias=True, dtype="f32", train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["switch", "fine", "large", "any", "any", "f32", "norm", "norm", "end", "end", "end_rows"])
    act, renorm, zipf = rng.choice(["relu", "swiglu"]), rng.randint(0, 1), round(rng.uniform(0.0, 1.5), 2)
    if kind == "switch":
        return dict(kind="few", T=_log_int(rng, 1, 64), d=768, F=3072, E=128, k=1, act="relu", dtype="bf16", renorm=0, shared_F=0, zipf=zipf)
    if kind == "fine":
        return dict(kind="few", T=_log_int(rng, 1, 32), d=2048, F=1408, E=60, k=4, act="swiglu", dtype="bf16", renorm=0, shared_F=5632, zipf=zipf)
    if kind == "large":
        return dict(kind="few", T=_log_int(rng, 1, 2), d=4096, F=14336, E=8, k=2, act="swiglu", dtype="bf16", renorm=1, shared_F=0, zipf=zipf)
    if kind == "any":       # widths, expert counts and activations in between
        E = rng.choice([4, 7, 16, 24, 48])
        return dict(kind="few", T=_log_int(rng, 1, 64), d=64 * _log_int(rng, 4, 32), F=64 * _log_int(rng, 8, 28), E=E, k=rng.randint(1, 4), act=act,
                    dtype="bf16", renorm=renorm, shared_F=rng.choice([0, 0, 64 * _log_int(rng, 8, 40)]), zipf=zipf)
    if kind == "f32":
        E = rng.choice([4, 8, 16, 32])
        return dict(kind="few", T=_log_int(rng, 1, 64), d=64 * _log_int(rng, 1, 16), F=64 * _log_int(rng, 2, 32), E=E, k=rng.randint(1, 2), act=act,
                    dtype="f32", renorm=renorm, shared_F=0, zipf=zipf)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    T = _log_int(rng, 1, 8192 if dtype == "bf16" else 4096)
    d = rng.choice([8 * _log_int(rng, 16, 512), 8 * _log_int(rng, 16, 512), _log_int(rng, 65, 4096)])
    if kind == "norm":
        return dict(kind="norm", T=T, d=d, norm=rng.choice(["rms", "layer"]), bias=rng.random() < 0.5, dtype=dtype, train=rng.random() < 0.6)
    case = dict(kind=kind, T=T, d=d, post=rng.choice(["none", "rms", "layer"]), gate=rng.choice(["none", "channel", "token"]),
                alpha=rng.choice([1.0, round(rng.uniform(0.5, 3.0), 2)]), next=rng.choice(["none", "rms", "layer"]), bias=rng.random() < 0.5,
                dtype=dtype, train=rng.random() < 0.6)
    if kind == "end_rows":
        return dict(case, train=False, T=_log_int(rng, 1, 4096), d=8 * _log_int(rng, 16, 256), k=rng.randint(1, 8), shared=rng.random() < 0.5)
    return case


# ------------------------------------------------------------------------------------ the inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _normal(shape, std, dtype, seed, stream, mean=0.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(mean, std, generator=torch.Generator(device=DEV).manual_seed(int(seed) * 64 + stream))


def _bias(E, s, seed):
    """A router bias that favours the experts by Zipf(s) shares over an order that the seed decides: the largest of E
    N(0,1) logits behaves like a choice by softmax at a temperature of 1 / sqrt(2 ln E)."""
    order = torch.randperm(E, generator=torch.Generator().manual_seed(int(seed)))
    return (-s * torch.log1p(order.double()) / math.sqrt(2.0 * math.log(E + 1.0))).float().to(DEV)


def _matrices(n, d, F, act, dtype, seed, stream):
    """Expert matrices in the paper's orientation: [n, inputs, outputs]."""
    names = (("W1", d, F), ("W2", F, d)) if act == "relu" else (("Wg", d, F), ("Wu", d, F), ("Wd", F, d))
    return {name: _normal((n, i, o), i ** -0.5, dtype, seed, stream + j) for j, (name, i, o) in enumerate(names)}


def _kernel_layout(w):
    """The matrices in the layout that moe_pack_weights and moe_pack_w_out document, and the tables of their addresses."""
    def rows(m):                       # [n, inputs, outputs] -> [n, blocks, 32, inputs]
        t = m.transpose(1, 2)
        t = t.reshape(t.shape[0], t.shape[1] // 32, 32, t.shape[2])
        return t if m.dtype == torch.float32 else torch.cat([t[:, :, 0::2], t[:, :, 1::2]], 2)

    first, last = (w["W1"], w["W2"]) if "W1" in w else (w["Wg"], w["Wd"])
    n, d, F = first.shape
    w_in = rows(first) if "W1" in w else torch.stack([rows(first), rows(w["Wu"])], 2)
    w_in, w_out = w_in.reshape(n, -1, d).contiguous(), rows(last).reshape(n, d, F).contiguous()
    w_out = w_out if first.dtype == torch.float32 else w_out.half()
    table = lambda t: t.data_ptr() + torch.arange(n, device=DEV) * (t[0].numel() * t.element_size())  # noqa: E731
    return {"w_in": w_in, "w_out": w_out, "in_ptrs": table(w_in), "out_ptrs": table(w_out)}


def _inputs(case, seed):
    T, d, dt, f32 = case["T"], case["d"], _dtype(case), torch.float32
    if case["kind"] == "few":
        got = {"x": _normal((T, d), 1.0, dt, seed, 1), "W_g": _normal((d, case["E"]), d ** -0.5, dt, seed, 2), "b": _bias(case["E"], case["zipf"], seed),
               "w": _matrices(case["E"], d, case["F"], case["act"], dt, seed, 20)}
        return dict(got, shared=_matrices(1, d, case["shared_F"], "swiglu", dt, seed, 30)) if case["shared_F"] else got
    vec = lambda stream: _normal((d,), 0.2, f32, seed, stream, 1.0)  # noqa: E731
    shift = lambda stream: _normal((d,), 0.2, f32, seed, stream) if case["bias"] else None  # noqa: E731
    # (the residual stream of a deep model: rows of different sizes, not centred)
    h = (_normal((T, d), 1.0, f32, seed, 1, 0.1) * _normal((T, 1), 0.5, f32, seed, 2, 2.0)).to(dt)
    if case["kind"] == "norm":
        return {"x": h, "w": vec(3), "b": shift(4), "du": _normal((T, d), 1.0, dt, seed, 5), "dx_add": _normal((T, d), 1.0, dt, seed, 6)}
    post, nxt = case["post"] != "none", case["next"] != "none"
    got = {"h": h, "post_w": vec(3) if post else None, "post_b": shift(4) if post else None, "next_w": vec(5) if nxt else None,
           "next_b": shift(6) if nxt else None,
           "gate": None if case["gate"] == "none" else _normal((1 if case["gate"] == "channel" else T, d), 0.3, f32, seed, 7, 0.5)}
    if case["kind"] == "end":
        return dict(got, v=_normal((T, d), 1.0, dt, seed, 8, 0.05), dy=_normal((T, d), 1.0, dt, seed, 9), du=_normal((T, d), 1.0, dt, seed, 10))
    A = T * case["k"]
    inv = torch.randperm(A, device=DEV, generator=torch.Generator(device=DEV).manual_seed(int(seed) * 64 + 11)).int()
    gate_w = torch.softmax(_normal((T, case["k"]), 1.0, f32, seed, 12), 1)
    return dict(got, y_perm=_normal((A, d), 1.0, f32, seed, 13), inv_perm=inv, gate_w=gate_w,
                shared=_normal((T, d), 1.0, f32, seed, 14) if case["shared"] else None)


def prepare(case, seed):
    """Inputs, the parameters as a program keeps them and, beside them, the buffers that it gives to the calls."""
    s, T, d, dt = dict(_inputs(case, seed), case=dict(case)), case["T"], case["d"], _dtype(case)
    new = lambda shape, t: torch.empty(shape, dtype=t, device=DEV)  # noqa: E731
    f32 = torch.float32
    if case["kind"] == "few":
        s.update(_kernel_layout(s["w"]), idx=new((T, case["k"]), torch.int32), gate_w=new((T, case["k"]), f32), y=new((T, d), dt))
        s["s_layout"] = _kernel_layout(s["shared"]) if case["shared_F"] else dict(in_ptrs=None, out_ptrs=None)
        s["W_gt"] = s["W_g"].t().contiguous()
        s["norm2"] = s["W_g"].double().square().sum(0).mul(1.000001).float()
        s["ws"] = new((T * (case["k"] * case["F"] + case["shared_F"]) * dt.itemsize,), torch.uint8)
    elif case["kind"] == "norm":
        s.update(u=new((T, d), dt), stats=new((T, 2), f32), dx=new((T, d), dt), dw=new((d,), f32), db=new((d,), f32) if case["bias"] else None,
                 ws=new((1024 * 2 * d,), f32))
    else:
        s.update(y=new((T, d), dt), u=None if case["next"] == "none" else new((T, d), dt), stats=new((T, 4), f32))
        if case["train"]:
            like = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731
            s.update(dv=new((T, d), dt), dh=new((T, d), dt), ws=new((1024 * 5 * d,), f32), dgate=like(s["gate"]),
                     **{"d" + n: like(s[n]) for n in ("post_w", "post_b", "next_w", "next_b")})
    return s


# ---------------------------------------------------------------------- the plain forms, in 32 bits
def _normed(x, kind, eps=1e-5):
    """n(x) and 1 / sqrt(...), in the type of x."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    r = 1.0 / (x.square().mean(1, keepdim=True) + eps).sqrt()
    return x * r, r


def _scaled(n, w, b):
    return n * w if b is None else n * w + b


def _norm_back(du, n, r, w, kind):
    """The gradient of the norm's input; dw, db."""
    g = du * w
    dx = g - n * (g * n).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - g.mean(1, keepdim=True)
    return dx * r, (du * n).sum(0), du.sum(0)


def _plain_norm(case, s, t):
    x, w, b = s["x"].to(t), s["w"].to(t), None if s["b"] is None else s["b"].to(t)
    n, r = _normed(x, case["norm"])
    out = {"u": _scaled(n, w, b)}
    if case["train"]:
        dx, dw, db = _norm_back(s["du"].to(t), n, r, w, case["norm"])
        out.update(dx=dx + s["dx_add"].to(t), dw=dw, db=db if case["bias"] else None)
    return out


def _plain_end(case, s, t, v):
    to = lambda n: None if s[n] is None else s[n].to(t)  # noqa: E731
    h, post_w, post_b, next_w, next_b, gate = (to(n) for n in ("h", "post_w", "post_b", "next_w", "next_b", "gate"))
    vn, vr = _normed(v, case["post"]) if case["post"] != "none" else (v, None)
    p = _scaled(vn, post_w, post_b) if case["post"] != "none" else v
    y = case["alpha"] * h + (p if gate is None else gate * p)
    yn, yr = _normed(y, case["next"]) if case["next"] != "none" else (None, None)
    out = {"y": y, "u": None if yn is None else _scaled(yn, next_w, next_b)}
    if case["train"]:
        gy = to("dy")
        if yn is not None:
            dn, out["dnext_w"], out["dnext_b"] = _norm_back(to("du"), yn, yr, next_w, case["next"])
            gy = gy + dn
        out["dh"] = case["alpha"] * gy
        dp = gy if gate is None else gate * gy
        if gate is not None:
            out["dgate"] = gy * p if case["gate"] == "token" else (gy * p).sum(0, keepdim=True)
        out["dv"] = dp
        if case["post"] != "none":
            out["dv"], out["dpost_w"], out["dpost_b"] = _norm_back(dp, vn, vr, post_w, case["post"])
        if not case["bias"]:
            out.update(dnext_b=None, dpost_b=None)
    return out


def _plain_rows(case, s, t):
    rows = s["y_perm"][s["inv_perm"].long()].to(t).reshape(case["T"], case["k"], case["d"])
    v = (rows * s["gate_w"].to(t)[:, :, None]).sum(1)
    return v if s["shared"] is None else v + s["shared"].to(t)


def _plain_ffn(x, w):
    """[n, T, d]: the product of every expert with every token."""
    if "W1" in w:
        return (x @ w["W1"].float()).clamp_min(0.0) @ w["W2"].float()
    g = x @ w["Wg"].float()
    return (g / (1.0 + torch.exp(-g)) * (x @ w["Wu"].float())) @ w["Wd"].float()


def _plain_few(case, s):
    x = s["x"].float()
    logits = x @ s["W_g"].float() + s["b"]
    idx = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :case["k"]]
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    gate = (e / e.sum(1, keepdim=True)).gather(1, idx)
    if case["renorm"]:
        gate = gate / gate.sum(1, keepdim=True)
    all_y = _plain_ffn(x, s["w"])
    y = (all_y[idx, torch.arange(case["T"], device=DEV)[:, None]] * gate[:, :, None]).sum(1)
    if case["shared_F"]:
        y = y + _plain_ffn(x, s["shared"])[0]
    return {"y": y, "idx": idx.int(), "gate_w": gate}


# -------------------------------------------------------------------------------------- one pass
def _run_plain(case, s):
    t = _dtype(case)
    if case["kind"] == "few":
        out = _plain_few(case, s)
        return dict(out, y=out["y"].to(t))
    if case["kind"] == "norm":
        out = _plain_norm(case, s, torch.float32)
    else:
        out = _plain_end(case, s, torch.float32, s["v"].float() if case["kind"] == "end" else _plain_rows(case, s, torch.float32))
    return {n: v.to(t) if v is not None and n in ("u", "dx", "y", "dv", "dh") else v for n, v in out.items()}


def _run_own(case, s):
    from paper_2506_12417_amd import binding as B
    T, d = case["T"], case["d"]
    dt = B.MOE_F32 if case["dtype"] == "f32" else B.MOE_BF16
    if case["kind"] == "few":
        act = B.MOE_SWIGLU if case["act"] == "swiglu" else B.MOE_RELU
        f32 = dt == B.MOE_F32
        B.moe_layer_few(s["x"], T, d, case["F"], case["E"], case["k"], act, dt, case["renorm"], s["W_g"] if f32 else s["W_gt"],
                        None if f32 else s["norm2"], s["b"], s["in_ptrs"], s["out_ptrs"], case["shared_F"], s["s_layout"]["in_ptrs"],
                        s["s_layout"]["out_ptrs"], s["idx"], s["gate_w"], s["ws"], s["ws"].numel(), s["y"], dt)
        return {n: s[n] for n in ("y", "idx", "gate_w")}
    if case["kind"] == "norm":
        kind, train = NORMS[case["norm"]], case["train"]
        B.moe_norm(s["x"], dt, s["w"], s["b"], T, d, kind, 1e-5, s["u"], dt, s["stats"] if train else None)
        if not train:
            return {"u": s["u"]}
        B.moe_norm_backward(s["du"], dt, s["x"], dt, s["w"], s["stats"], T, d, kind, s["dx_add"], s["dx"], s["dw"], s["db"], s["ws"],
                            s["ws"].numel() * 4)
        return {n: s[n] for n in ("u", "dx", "dw", "db")}
    post, nxt = NORMS[case["post"]], NORMS[case["next"]]
    gate_rows = {"none": 0, "channel": 1, "token": T}[case["gate"]]
    norms = (post, 1e-5, s["post_w"], s["post_b"], s["gate"], gate_rows, case["alpha"], nxt, 1e-5, s["next_w"], s["next_b"])
    if case["kind"] == "end_rows":
        B.moe_block_end_rows(s["y_perm"], s["inv_perm"], s["gate_w"], s["shared"], case["k"], s["h"], dt, T, d, *norms, s["y"], s["u"], dt)
        return {n: s[n] for n in ("y", "u")}
    B.moe_block_end(s["v"], dt, s["h"], dt, T, d, *norms, s["y"], s["u"], dt, s["stats"] if case["train"] else None)
    if not case["train"]:
        return {n: s[n] for n in ("y", "u")}
    B.moe_block_end_backward(s["dy"], s["du"] if nxt else None, dt, s["v"], dt, s["h"], dt, T, d, post, s["post_w"], s["post_b"], s["gate"],
                             gate_rows, case["alpha"], nxt, s["next_w"], s["stats"], s["dv"], s["dh"], s["dpost_w"], s["dpost_b"], s["dgate"],
                             s["dnext_w"], s["dnext_b"], s["ws"], s["ws"].numel() * 4)
    return {n: s[n] for n in ("y", "u", "dv", "dh", "dgate", "dpost_w", "dpost_b", "dnext_w", "dnext_b")}


def run(state):
    return (_run_own if own else _run_plain)(state["case"], state)


# ------------------------------------------------------------------------- what a pass must cost
def work(case):
    T, d, es = case["T"], case["d"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "few":
        E, k, F, mats = case["E"], case["k"], case["F"], 2 if case["act"] == "relu" else 3
        p = [(i + 1.0) ** -case["zipf"] for i in range(E)]
        active = sum(1.0 - (1.0 - v / sum(p)) ** (T * k) for v in p)      # experts that T k draws from the shares hit
        active = min(max(active, k), E)
        return {"bytes": 2 * T * d * es + d * E * es + 4 * E + 8 * T * k + active * mats * d * F * es + 3 * d * case["shared_F"] * es,
                "flops": 2 * T * d * E + 2 * T * k * d * F * mats + 6 * T * d * case["shared_F"]}
    n, vecs = T * d, sum(case.get(name, "none") != "none" for name in ("norm", "post", "next")) * (2 if case["bias"] else 1)
    if case["kind"] == "norm":
        return {"bytes": n * es * (5 if case["train"] else 2) + 4 * d * vecs * (2 if case["train"] else 1), "flops": n * (16 if case["train"] else 5)}
    gate = {"none": 0, "channel": d, "token": n}[case["gate"]]
    outs = 1 + (case["next"] != "none")
    small = 4 * d * vecs + 4 * gate
    if case["kind"] == "end_rows":
        A = T * case["k"]
        return {"bytes": 4 * n * (case["k"] + case["shared"]) + 8 * A + n * es * (1 + outs) + small, "flops": n * (2 * case["k"] + 12)}
    # (a training step reads v, h, dy and du once and writes y, u, dv and dh)
    if case["train"]:
        return {"bytes": n * es * (2 + 1 + 2 + 2 * (outs - 1) + 1) + 2 * small, "flops": n * 40}
    return {"bytes": n * es * (2 + outs) + small, "flops": n * 12}


# --------------------------------------------------------------------- the same in 64 bits, plainly
def _exact_norm(x, kind):
    mean = x.sum(1) / x.shape[1] if kind == "layer" else torch.zeros_like(x[:, 0])
    var = ((x - mean[:, None]) ** 2).sum(1) / x.shape[1]
    r = (var + 1e-5) ** -0.5
    return (x - mean[:, None]) * r[:, None], r


def _exact_norm_back(g, n, r, kind):
    """The norm's derivative applied to the gradient g of n: the projection away from n (and from the ones), times r."""
    d = n.shape[1]
    out = g - n * (torch.linalg.vecdot(g, n) / d)[:, None]
    return (out - (g.sum(1) / d)[:, None] if kind == "layer" else out) * r[:, None]


def exact(case, seed):
    s = _inputs(case, seed)
    s = {n: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for n, v in s.items()}
    if case["kind"] == "few":
        x, k = s["x"], case["k"]
        logits = x @ s["W_g"] + s["b"]
        top, idx = torch.topk(logits, k, dim=1)
        gate = torch.exp(top - torch.logsumexp(top if case["renorm"] else logits, 1, keepdim=True))
        y = torch.zeros_like(x)
        jobs = [(s["w"], e, *(idx == e).nonzero(as_tuple=True)) for e in range(case["E"])]
        if case["shared_F"]:
            jobs.append((s["shared"], 0, torch.arange(case["T"], device=DEV), None))
        for w, e, t, j in jobs:
            if t.numel():
                m = {n: a[e].double() for n, a in w.items()}
                hid = torch.relu(x[t] @ m["W1"]) if "W1" in m else torch.nn.functional.silu(x[t] @ m["Wg"]) * (x[t] @ m["Wu"])
                o = hid @ (m["W2"] if "W2" in m else m["Wd"])
                y.index_add_(0, t, o if j is None else o * gate[t, j][:, None])
        return {"y": y, "idx": idx.int(), "gate_w": gate}
    if case["kind"] == "norm":
        n, r = _exact_norm(s["x"], case["norm"])
        out = {"u": n * s["w"] + (s["b"] if case["bias"] else 0.0)}
        if case["train"]:
            out.update(dx=_exact_norm_back(s["du"] * s["w"], n, r, case["norm"]) + s["dx_add"], dw=torch.linalg.vecdot(s["du"], n, dim=0),
                       db=s["du"].sum(0) if case["bias"] else None)
        return out
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    pb, nb = (zero if s[n] is None else s[n] for n in ("post_b", "next_b"))
    gate = zero + 1.0 if s["gate"] is None else s["gate"]
    if case["kind"] == "end":
        v = s["v"]
    else:
        inv = s["inv_perm"].long().reshape(case["T"], case["k"])
        v = zero + (0.0 if s["shared"] is None else s["shared"])
        for j in range(case["k"]):
            v = v + s["gate_w"][:, j, None] * s["y_perm"][inv[:, j]]
    p, post, nxt = v, case["post"] != "none", case["next"] != "none"
    if post:
        vn, vr = _exact_norm(v, case["post"])
        p = vn * s["post_w"] + pb
    y = case["alpha"] * s["h"] + gate * p
    out = {"y": y, "u": None}
    if nxt:
        yn, yr = _exact_norm(y, case["next"])
        out["u"] = yn * s["next_w"] + nb
    if case["train"]:
        gy = s["dy"] + (_exact_norm_back(s["du"] * s["next_w"], yn, yr, case["next"]) if nxt else 0.0)
        gv = gate * gy
        out.update(dh=case["alpha"] * gy, dv=_exact_norm_back(gv * s["post_w"], vn, vr, case["post"]) if post else gv)
        out["dgate"] = None if s["gate"] is None else gy * p if case["gate"] == "token" else (gy * p).sum(0, keepdim=True)
        for name, on, g, n in (("next", nxt, s["du"], yn if nxt else None), ("post", post, gv, vn if post else None)):
            out["d" + name + "_w"] = torch.linalg.vecdot(g, n, dim=0) if on else None
            out["d" + name + "_b"] = g.sum(0) if on and case["bias"] else None
    return out
