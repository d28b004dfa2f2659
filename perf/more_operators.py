"""Performance cases of a MoE layer's training step: hidden activations kept in 8 bits for the backward pass, the experts' gradients made
from them, the gradients of the token sort and of the weighted combine, and the router's.

Kinds of case:

  keep    the experts' first product, which keeps the pre-activations in 8 bits beside its output, and their values read back
  rows    any rows of activations put into that format and read back
  back    the gradients of the experts (weights, input, gate values) from what was kept, and the sum over a token's rows
  sort    the gradients of the combine (rows weighted, gate values) and of the sort (a token's rows added up), each on its own
  route   the router's gradients: logits, input, matrix and bias

All inputs are drawn on the GPU from the seed alone: activations and gradients N(0,1), matrices N(0,1/fan_in), experts chosen with roughly
Zipf-distributed loads.  Plain form: elementary torch operations in 32 bits, one product an expert where experts have rows of their own.
"""
import math

import torch

own = False
DEV = "cuda:0"
BLOCK = 64          # columns that share a scale


# ------------------------------------------------------------------------------------- the cases
def listed():
    switch = dict(d=768, F=3072, E=128, k=1, act="relu", zipf=1.0)
    fine = dict(d=2048, F=1408, E=60, k=4, act="swiglu", zipf=1.2)
    large = dict(d=4096, F=14336, E=8, k=2, act="swiglu", zipf=2.0)
    return [
        # a short sequence through many small experts: the fetch of the weights and latencies
        dict(switch, name="keep_short", kind="keep", T=100),
        # a training step's first product at the benchmark's sizes
        dict(fine, name="keep_fine", kind="keep", T=8192),
        # a block's output, kept for the gradient of the norm behind it
        dict(name="rows_train", kind="rows", rows=8192, n=2048, dtype="f32"),
        # a width that is no multiple of anything
        dict(name="rows_odd", kind="rows", rows=1501, n=777, dtype="bf16"),
        # the experts' gradients over a short sequence: most experts have no row, all matrices' gradients are written
        dict(switch, name="back_short", kind="back", T=100),
        # training steps at the benchmark's sizes: top-1 over many experts, fine-grained experts, large and very skewed ones
        dict(switch, name="back_switch", kind="back", T=16384),
        dict(fine, name="back_fine", kind="back", T=8192),
        dict(large, name="back_large", kind="back", T=8192),
        # gradients of the dispatch of a rank whose experts run elsewhere
        dict(name="sort_fine", kind="sort", T=8192, d=2048, k=4, dtype="bf16"),
        # fp32 and a ragged width
        dict(name="sort_odd", kind="sort", T=1501, d=777, k=3, dtype="f32"),
        # the routers: softmax over many experts, top-1; a layer kept in fp32 with renormalised gates
        dict(name="route_switch", kind="route", T=16384, d=768, E=128, k=1, renorm=0, dtype="bf16"),
        dict(name="route_f32", kind="route", T=1501, d=1032, E=60, k=4, renorm=1, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["keep", "keep", "rows", "back", "back", "back", "sort", "route"])
    if kind == "rows":
        return dict(kind="rows", rows=_log_int(rng, 1, 16384), n=rng.choice([64 * _log_int(rng, 1, 64), _log_int(rng, 1, 4096)]),
                    dtype=rng.choice(["f32", "bf16"]))
    if kind == "sort":
        return dict(kind="sort", T=_log_int(rng, 1, 8192), d=rng.choice([8 * _log_int(rng, 8, 256), _log_int(rng, 65, 2048)]), k=rng.randint(1, 8),
                    dtype=rng.choice(["f32", "bf16"]))
    if kind == "route":
        renorm = rng.randint(0, 1)
        E = _log_int(rng, 4, 256)
        return dict(kind="route", T=_log_int(rng, 1, 16384), d=8 * _log_int(rng, 16, 256), E=E, k=rng.randint(1 + renorm, min(E, 8)), renorm=renorm,
                    dtype=rng.choice(["f32", "bf16", "bf16"]))
    shape = rng.choice(["switch", "fine", "any", "any"])
    T, zipf = _log_int(rng, 1, 8192), round(rng.uniform(0.0, 1.5), 2)
    if shape == "switch":
        return dict(kind=kind, T=T, d=768, F=3072, E=128, k=1, act="relu", zipf=zipf)
    if shape == "fine":
        return dict(kind=kind, T=T, d=2048, F=1408, E=60, k=4, act="swiglu", zipf=zipf)
    E = rng.choice([1, 4, 7, 16, 24, 48])
    return dict(kind=kind, T=T, d=64 * _log_int(rng, 4, 40), F=64 * _log_int(rng, 4, 56), E=E, k=rng.randint(1, min(E, 4)),
                act=rng.choice(["relu", "swiglu"]), zipf=zipf)


# ------------------------------------------------------------------------------------ the inputs
def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _normal(shape, std, dtype, seed, stream, mean=0.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(mean, std, generator=torch.Generator(device=DEV).manual_seed(int(seed) * 64 + stream))


def _routing(case, seed):
    """Which experts the tokens chose (k of E without repeats, loads roughly by Zipf), their gate values and the sort by expert."""
    T, E, k = case["T"], case["E"], case["k"]
    order = torch.randperm(E, generator=torch.Generator().manual_seed(int(seed)))
    score = (-case["zipf"] * torch.log1p(order.double())).float().to(DEV)
    u = torch.empty((T, E), device=DEV).exponential_(1.0, generator=torch.Generator(device=DEV).manual_seed(int(seed) * 64 + 3))
    idx = torch.topk(score - u.log(), k, dim=1)[1].int()
    gate_w = torch.softmax(_normal((T, k), 1.0, torch.float32, seed, 4), 1) * (0.9 if k > 1 else 0.3)
    perm = torch.sort(idx.reshape(-1), stable=True)[1].int()
    inv = torch.empty_like(perm)
    inv[perm.long()] = torch.arange(T * k, device=DEV, dtype=torch.int32)
    counts = torch.bincount(idx.reshape(-1), minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = counts.cumsum(0).int()
    return {"gate_w": gate_w, "perm": perm, "inv_perm": inv, "offsets": offsets, "counts": counts.tolist()}


def _matrices(case, seed):
    """The experts' matrices as a training program has them: [E, inputs, outputs]."""
    E, d, F, t = case["E"], case["d"], case["F"], torch.bfloat16
    w = {"a": _normal((E, d, F), d ** -0.5, t, seed, 20), "o": _normal((E, F, d), F ** -0.5, t, seed, 22)}
    return dict(w, b=_normal((E, d, F), d ** -0.5, t, seed, 21)) if case["act"] == "swiglu" else w


def _blocks(x):
    """[rows, n] -> [rows, blocks, 64], the last block filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK)).reshape(x.shape[0], -(-x.shape[1] // BLOCK), BLOCK)


def _quantised(z, positive):
    """8-bit values and a scale for every 64 columns of a row.  positive: what is above zero stays above zero."""
    b = _blocks(z)
    most = b.abs().amax(2, keepdim=True)
    q = torch.where(most > 0, (b * (127.0 / most)).round(), 0.0)
    if positive:
        q = torch.where(b > 0, q.clamp_min(1.0), 0.0)
    return q.flatten(1)[:, :z.shape[1]].to(torch.int8).contiguous(), (most[:, :, 0] / 127.0).contiguous()


def _inputs(case, seed):
    f32, bf16, kind = torch.float32, torch.bfloat16, case["kind"]
    if kind == "rows":
        return {"x": (_normal((case["rows"], case["n"]), 1.0, f32, seed, 1, 0.1) * _normal((case["rows"], 1), 0.5, f32, seed, 2, 2.0)).to(_dtype(case))}
    T, d, k, dt = case["T"], case["d"], case["k"], _dtype(case)
    if kind == "sort":
        A = T * k
        inv = torch.randperm(A, device=DEV, generator=torch.Generator(device=DEV).manual_seed(int(seed) * 64 + 1)).int()
        return {"dy": _normal((T, d), 1.0, dt, seed, 2), "y_perm": _normal((A, d), 1.0, f32, seed, 5), "inv_perm": inv,
                "gate_w": torch.softmax(_normal((T, k), 1.0, f32, seed, 6), 1), "dx_perm": _normal((A, d), 1.0, f32, seed, 7),
                "dx_add": _normal((T, d), 1.0, f32, seed, 8)}
    if kind == "route":
        E = case["E"]
        logits = _normal((T, E), 1.0, f32, seed, 2)
        top, idx = torch.topk(logits, k, dim=1)
        gate_w = torch.exp(top - torch.logsumexp(top if case["renorm"] else logits, 1, keepdim=True))
        return {"x": _normal((T, d), 1.0, dt, seed, 5), "W_g": _normal((d, E), d ** -0.5, dt, seed, 6), "logits": logits, "idx": idx.int(),
                "gate_w": gate_w, "dgate_w": _normal((T, k), 1.0, f32, seed, 7), "dx_add": _normal((T, d), 0.1, f32, seed, 8)}
    s = dict(_routing(case, seed), x=_normal((T, d), 1.0, bf16, seed, 1), w=_matrices(case, seed))
    if kind == "back":
        s["dy"] = _normal((T, d), 1.0, bf16, seed, 2)
        z = _normal((T * k, case["F"] * (2 if case["act"] == "swiglu" else 1)), 1.0, f32, seed, 5)
        s["z_q"], s["z_scale"] = _quantised(z, case["act"] == "relu")
    return s


def _packed_in(w):
    """The first matrices in the layout that moe_pack_weights documents."""
    def rows(m):                       # [E, inputs, outputs] -> [E, blocks, 32, inputs]
        t = m.transpose(1, 2)
        t = t.reshape(t.shape[0], t.shape[1] // 32, 32, t.shape[2])
        return torch.cat([t[:, :, 0::2], t[:, :, 1::2]], 2)

    E, d, _ = w["a"].shape
    return (torch.stack([rows(w["a"]), rows(w["b"])], 2) if "b" in w else rows(w["a"])).reshape(E, -1, d).contiguous()


def prepare(case, seed):
    """Inputs and what a program keeps beside them: packed weights, and the buffers that it gives to the calls."""
    s, kind = dict(_inputs(case, seed), case=dict(case)), case["kind"]
    new = lambda shape, t: torch.empty(shape, dtype=t, device=DEV)  # noqa: E731
    f32, bf16 = torch.float32, torch.bfloat16
    if kind == "rows":
        rows, n = case["rows"], case["n"]
        return dict(s, q=new((rows, n), torch.int8), scale=new((rows, -(-n // BLOCK)), f32), back=new((rows, n), bf16))
    T, d, k, dt = case["T"], case["d"], case["k"], _dtype(case)
    if kind == "sort":
        return dict(s, dy_perm=new((T * k, d), dt), dgate_w=new((T, k), f32), dx=new((T, d), dt))
    if kind == "route":
        E = case["E"]
        return dict(s, dlogits=new((T, E), f32), dx=new((T, d), f32), dw=new((d, E), f32), db=new((E,), f32), ws=new((64 << 20,), torch.uint8))
    A, E, F, w = T * k, case["E"], case["F"], s["w"]
    Z = F * (2 if case["act"] == "swiglu" else 1)
    if kind == "keep":
        s["w_in"] = _packed_in(w)
        del w["o"]
        s["in_ptrs"] = s["w_in"].data_ptr() + torch.arange(E, device=DEV) * (Z * d * 2)
        return dict(s, h=new((A, F), torch.float16), z_q=new((A, Z), torch.int8), z_scale=new((A, Z // BLOCK), f32), z=new((A, Z), bf16))
    like = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731
    # (room for the gradients of the hidden activations and the weighted activations, and a little for sums)
    ws = new((A * (Z + F) * 2 + A * 4 * (-(-F // 64)) + (1 << 20),), torch.uint8)
    return dict(s, dw={n: like(w.get(n)) for n in "abo"}, dx_perm=new((A, d), f32), dgate_w=new((T, k), f32), dx=new((T, d), bf16), ws=ws)


# ---------------------------------------------------------------------- the plain forms, in 32 bits
def _restored(q, scale):
    return (_blocks(q.float()) * scale[:, :, None]).flatten(1)[:, :q.shape[1]]


def _sorted_rows(s, name):
    """The tokens' rows in the experts' order, an expert's at a time."""
    case = s["case"]
    return s[name].float()[s["perm"].long() // case["k"]].split(s["counts"])


def _plain_keep(case, s):
    w = s["w"]
    z = torch.cat([torch.cat([x @ w[n][e].float() for n in "ab" if n in w], 1) for e, x in enumerate(_sorted_rows(s, "x"))])
    if case["act"] == "relu":
        h = z.clamp_min(0.0)
        q, scale = _quantised(h, True)
    else:
        g, u = z.chunk(2, 1)
        h = g / (1.0 + torch.exp(-g)) * u
        q, scale = _quantised(z, False)
    return {"h": h.half(), "z": _restored(q, scale).bfloat16()}


def _plain_back(case, s):
    w, bf16 = s["w"], torch.bfloat16
    xs, dys = _sorted_rows(s, "x"), _sorted_rows(s, "dy")
    gate = s["gate_w"].reshape(-1)[s["perm"].long()].split(s["counts"])
    q, scale = s["z_q"].split(s["counts"]), s["z_scale"].split(s["counts"])
    dx_rows, dgate, dw = [], [], {n: torch.empty_like(m) for n, m in w.items()}
    for e in range(case["E"]):
        z = _restored(q[e], scale[e])
        grad_h = dys[e] @ w["o"][e].float().t()
        if case["act"] == "relu":
            h, dz = z, [gate[e][:, None] * grad_h * (q[e] > 0)]
        else:
            g, u = z.chunk(2, 1)
            sig = 1.0 / (1.0 + torch.exp(-g))
            h, dh = g * sig * u, gate[e][:, None] * grad_h
            dz = [dh * u * sig * (1.0 + g * (1.0 - sig)), dh * g * sig]
        dgate.append((h * grad_h).sum(1))
        dw["o"][e] = ((gate[e][:, None] * h).t() @ dys[e]).to(bf16)
        for n, grad in zip("ab", dz):
            dw[n][e] = (xs[e].t() @ grad).to(bf16)
        dx_rows.append(sum(grad @ w[n][e].float().t() for n, grad in zip("ab", dz)))
    inv = s["inv_perm"].long()
    dx = torch.cat(dx_rows)[inv].reshape(case["T"], case["k"], case["d"]).sum(1)
    return {"dx": dx.to(bf16), "dgate_w": torch.cat(dgate)[inv].reshape(case["T"], case["k"]), "dw": dw}


def _plain_sort(case, s):
    T, d, k, t = case["T"], case["d"], case["k"], _dtype(case)
    inv, dy = s["inv_perm"].long(), s["dy"].float()
    rows = s["y_perm"][inv].reshape(T, k, d)
    dy_perm = torch.empty((T * k, d), dtype=t, device=DEV)
    dy_perm[inv] = (s["gate_w"][:, :, None] * dy[:, None]).to(t).reshape(T * k, d)
    dx = s["dx_add"] + s["dx_perm"][inv].reshape(T, k, d).sum(1)
    return {"dy_perm": dy_perm, "dgate_w": (rows * dy[:, None]).sum(2), "dx": dx.to(t)}


def _plain_route(case, s):
    idx, g, dg = s["idx"].long(), s["gate_w"], s["dgate_w"]
    dot = (g * dg).sum(1, keepdim=True)
    if case["renorm"]:
        dl = torch.zeros_like(s["logits"]).scatter(1, idx, g * (dg - dot))
    else:
        e = torch.exp(s["logits"] - s["logits"].amax(1, keepdim=True))
        dl = e / e.sum(1, keepdim=True) * (torch.zeros_like(e).scatter(1, idx, dg) - dot)
    return {"dlogits": dl, "dx": s["dx_add"] + dl @ s["W_g"].float().t(), "dw": s["x"].float().t() @ dl, "db": dl.sum(0)}


# -------------------------------------------------------------------------------------- one pass
def _run_plain(case, s):
    if case["kind"] == "rows":
        return {"x": _restored(*_quantised(s["x"].float(), False)).bfloat16()}
    return {"keep": _plain_keep, "back": _plain_back, "sort": _plain_sort, "route": _plain_route}[case["kind"]](case, s)


def _run_own(case, s):
    from paper_2506_12417_amd import binding as B
    dt, kind = B.MOE_F32 if case.get("dtype") == "f32" else B.MOE_BF16, case["kind"]
    if kind == "rows":
        rows, n = case["rows"], case["n"]
        B.moe_keep_rows(s["x"], dt, rows, n, s["q"], s["scale"])
        B.moe_keep_restore(s["q"], s["scale"], rows, n, s["back"], B.MOE_BF16)
        return {"x": s["back"]}
    T, d, k = case["T"], case["d"], case["k"]
    if kind == "sort":
        B.moe_unpermute_combine_backward(s["dy"], dt, s["y_perm"], s["inv_perm"], s["gate_w"], T, d, k, s["dy_perm"], dt, s["dgate_w"])
        B.moe_permute_backward(s["dx_perm"], s["inv_perm"], T, d, k, s["dx_add"], s["dx"], dt)
        return {n: s[n] for n in ("dy_perm", "dgate_w", "dx")}
    if kind == "route":
        B.moe_route_topk_backward(s["dgate_w"], s["gate_w"], s["idx"], s["logits"], None, s["x"], s["W_g"], T, d, case["E"], k, case["renorm"], dt,
                                  s["dlogits"], s["dx_add"], s["dx"], s["dw"], s["db"], s["ws"], s["ws"].numel())
        return {n: s[n] for n in ("dlogits", "dx", "dw", "db")}
    F, E, act = case["F"], case["E"], B.MOE_SWIGLU if case["act"] == "swiglu" else B.MOE_RELU
    if kind == "keep":
        B.moe_grouped_ffn_keep(s["x"], T, d, F, E, k, act, dt, s["in_ptrs"], s["offsets"], s["perm"], s["h"], s["z_q"], s["z_scale"])
        B.moe_keep_restore(s["z_q"], s["z_scale"], T * k, s["z_q"].shape[1], s["z"], dt)
        return {n: s[n] for n in ("h", "z")}
    w, dw = s["w"], s["dw"]
    B.moe_grouped_ffn_backward(s["dy"], dt, s["x"], T, d, F, E, k, act, dt, w["a"], w.get("b"), w["o"], s["offsets"], s["perm"], s["inv_perm"],
                               s["gate_w"], s["z_q"], s["z_scale"], s["dx_perm"], s["dgate_w"], dw["a"], dw["b"], dw["o"], dt, 0, s["ws"],
                               s["ws"].numel())
    B.moe_permute_backward(s["dx_perm"], s["inv_perm"], T, d, k, None, s["dx"], dt)
    return {"dx": s["dx"], "dgate_w": s["dgate_w"], "dw": {n: m for n, m in dw.items() if m is not None}}


def run(state):
    return (_run_own if own else _run_plain)(state["case"], state)


# ------------------------------------------------------------------------- what a pass must cost
def work(case):
    kind, es = case["kind"], 4 if case.get("dtype") == "f32" else 2
    if kind == "rows":
        n = case["rows"] * case["n"]
        return {"bytes": n * (es + 1 + 1 + 2) + 2 * 4 * case["rows"] * -(-case["n"] // BLOCK), "flops": 4 * n}
    T, d, k = case["T"], case["d"], case["k"]
    A = T * k
    if kind == "sort":
        return {"bytes": T * d * (es + 4 + es) + A * d * (4 + es + 4) + A * 16, "flops": A * d * 4}
    if kind == "route":
        E = case["E"]
        return {"bytes": T * d * (es + 8) + T * E * (4 + (0 if case["renorm"] else 4)) + T * k * 12 + d * E * (es + 4), "flops": 4 * T * d * E}
    E, F, mats = case["E"], case["F"], 2 if case["act"] == "relu" else 3
    Z = F * (mats - 1)
    p = [(i + 1.0) ** -case["zipf"] for i in range(E)]
    active = min(max(sum(1.0 - (1.0 - v / sum(p)) ** A for v in p), k), E)      # experts that A draws from the shares hit
    if kind == "keep":
        # (what is kept is written, and read again where its values are wanted)
        return {"bytes": T * d * 2 + active * d * Z * 2 + A * F * 2 + A * Z * 4 + A * Z // 8 + 4 * A, "flops": 2 * A * d * Z}
    return {"bytes": 3 * T * d * 2 + A * Z + A * Z // 16 + 16 * A + (active + E) * mats * d * F * 2, "flops": 4 * A * d * F * mats}


# --------------------------------------------------------------------- the same in 64 bits, plainly
def _exact_values(q, scale):
    return q.double() * scale.double().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _exact_kept(z, positive):
    rows, n = z.shape
    padded = torch.zeros((rows, -(-n // BLOCK) * BLOCK), dtype=torch.float64, device=DEV)
    padded[:, :n] = z
    step = padded.abs().reshape(rows, -1, BLOCK).max(2)[0].repeat_interleave(BLOCK, 1) / 127.0
    near = torch.round(padded / step.clamp_min(1e-300))
    if positive:
        near = torch.maximum(near, torch.sign(padded))
    return (near * step)[:, :n]


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "rows":
        return {"x": _exact_kept(s["x"].double(), False)}
    T, d, k = case["T"], case["d"], case["k"]
    if kind == "sort":
        inv, dy = s["inv_perm"].long(), s["dy"].double()
        back = torch.empty_like(inv)
        back[inv] = torch.arange(T * k, device=DEV)                  # sorted row -> assignment
        at = back // k
        dgate = torch.empty(T * k, dtype=torch.float64, device=DEV)
        dgate[back] = torch.linalg.vecdot(dy[at], s["y_perm"].double())
        return {"dy_perm": dy[at] * s["gate_w"].double().reshape(-1)[back][:, None], "dgate_w": dgate.reshape(T, k),
                "dx": s["dx_add"].double().index_add(0, at, s["dx_perm"].double())}
    if kind == "route":
        logits, idx = s["logits"].double().requires_grad_(), s["idx"].long()
        gate = torch.gather(logits, 1, idx).softmax(1) if case["renorm"] else torch.gather(logits.softmax(1), 1, idx)
        dl, = torch.autograd.grad(gate, logits, s["dgate_w"].double())
        return {"dlogits": dl, "dx": torch.addmm(s["dx_add"].double(), dl, s["W_g"].double().t()), "dw": torch.mm(s["x"].double().t(), dl),
                "db": torch.mv(dl.t(), torch.ones(T, dtype=torch.float64, device=DEV))}
    w, perm, bounds = s["w"], s["perm"].long(), s["offsets"].tolist()
    relu, F = case["act"] == "relu", case["F"]
    if kind == "keep":
        h, z = [], []
        for e in range(case["E"]):
            x = s["x"][perm[bounds[e]:bounds[e + 1]] // k].double()
            g = torch.mm(x, w["a"][e].double())
            u = None if relu else torch.mm(x, w["b"][e].double())
            h.append(torch.relu(g) if relu else torch.nn.functional.silu(g) * u)
            z.append(torch.relu(g) if relu else torch.hstack([g, u]))
        return {"h": torch.vstack(h), "z": _exact_kept(torch.vstack(z), relu)}
    dx = torch.zeros((T, d), dtype=torch.float64, device=DEV)
    dgate = torch.zeros(T * k, dtype=torch.float64, device=DEV)
    dw = {n: torch.zeros(m.shape, dtype=torch.float64, device=DEV) for n, m in w.items()}
    gates = s["gate_w"].double().reshape(-1)
    for e in range(case["E"]):
        a = perm[bounds[e]:bounds[e + 1]]
        if not a.numel():
            continue
        x, dy, z = s["x"][a // k].double(), s["dy"][a // k].double(), _exact_values(s["z_q"][bounds[e]:bounds[e + 1]], s["z_scale"][bounds[e]:bounds[e + 1]])
        z.requires_grad_()
        out, weight = w["o"][e].double().requires_grad_(), gates[a].requires_grad_()
        # (a value that was kept above zero is one where the ReLU has slope 1)
        hidden = torch.relu(z) if relu else torch.nn.functional.silu(z[:, :F]) * z[:, F:]
        dz, dw["o"][e], dgate[a] = torch.autograd.grad(weight[:, None] * torch.mm(hidden, out), (z, out, weight), dy)
        for n, part in zip("ab", dz.split(F, 1)):
            dw[n][e] = torch.mm(x.t(), part)
            dx.index_add_(0, a // k, torch.mm(part, w[n][e].double().t()))
    return {"dx": dx, "dgate_w": dgate.reshape(T, k), "dw": dw}
