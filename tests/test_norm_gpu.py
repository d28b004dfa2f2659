"""moe_norm, moe_block_end, moe_block_end_rows and their gradients against the formulas in 64 bits.

Tolerance.  Every quantity of the reference carries a magnitude: what its terms add up to in absolute value, errors of
its inputs passed on (the mean's, the mean square's, the sums' of the backward formulas).  A chain of fp32 operations is off
by at most about as many units (2^-24) of that magnitude as it has roundings in a row.  A row's sum has up to 8 in a
thread, 4 + 3 across lanes and 4 + 3 across wavefronts, and three such sums stand behind one another with a dozen
elementwise operations between: below 96.  A parameter's gradient adds up to ceil(T / 1024) rows in a thread and 64 + 16 parts.  The
outputs' own rounding comes on top: half a unit of their type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

UNITS = 96 * 2.0 ** -24
NONE, RMS, LAYER = 0, 1, 2
F32, BF16 = 0, 1
EPS = 1e-5


def _torch():
    import torch
    from paper_2506_12417_amd import binding as B
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return torch, B


class Num:
    """A value in 64 bits and the magnitude of what it was made of."""

    def __init__(self, v, mag=None):
        self.v = np.asarray(v, dtype=np.float64)
        self.m = np.abs(self.v) if mag is None else mag

    def __add__(self, o):
        return Num(self.v + o.v, self.m + o.m)

    def __sub__(self, o):
        return Num(self.v - o.v, self.m + o.m)

    def __mul__(self, o):
        return Num(self.v * o.v, np.maximum(self.m * np.abs(o.v) + np.abs(self.v) * o.m, np.abs(self.v * o.v)))

    def mean(self):
        return Num(self.v.mean(1, keepdims=True), self.m.mean(1, keepdims=True))

    def total(self):
        return Num(self.v.sum(0), self.m.sum(0))


def norm(x, kind, eps=EPS):
    """n(x) and r as Nums."""
    if kind == LAYER:
        x = x - x.mean()
    sq = (x * x).mean()
    r = 1.0 / np.sqrt(sq.v + eps)
    r = Num(r, r + 0.5 * sq.m * r ** 3)
    return x * r, r


def scaled(n, w, b):
    if w is not None:
        n = n * Num(w)
    return n if b is None else n + Num(b)


def norm_back(g, n, r, kind):
    out = g - n * (g * n).mean()
    if kind == LAYER:
        out = out - g.mean()
    return out * r


def reference(a):
    """All outputs of a block's end (and its gradients) for the inputs in the dict a; v is None for moe_norm alone."""
    h, out, vn, vr = Num(a["h"]), {}, None, None
    y = h
    if a["v"] is not None:
        v = Num(a["v"])
        vn = v
        if a["post"] != NONE:
            vn, vr = norm(v, a["post"])
        p = scaled(vn, a["post_w"], a["post_b"]) if a["post"] != NONE else v
        y = Num(a["alpha"]) * h + (p if a["gate"] is None else Num(a["gate"]) * p)
        out["y"] = y
    if a["next"] != NONE:
        yn, yr = norm(y, a["next"])
        out["u"] = scaled(yn, a["next_w"], a["next_b"])
    if a["dy"] is None and a["du"] is None:
        return out
    gy = Num(np.zeros_like(a["h"])) if a["dy"] is None else Num(a["dy"])
    if a["du"] is not None:
        du = Num(a["du"])
        out["dnext_w"], out["dnext_b"] = (du * yn).total(), du.total()
        gy = gy + norm_back(du if a["next_w"] is None else du * Num(a["next_w"]), yn, yr, a["next"])
    out["dh"] = Num(a["alpha"]) * gy if a["v"] is not None else gy
    if a["v"] is not None:
        if a["gate"] is not None:
            dg = gy * p
            out["dgate"] = dg if a["gate"].shape[0] == a["h"].shape[0] and a["h"].shape[0] > 1 else Num(dg.v.sum(0, keepdims=True), dg.m.sum(0, keepdims=True))
        dp = gy if a["gate"] is None else gy * Num(a["gate"])
        out["dv"] = dp
        if a["post"] != NONE:
            out["dpost_w"], out["dpost_b"] = (dp * vn).total(), dp.total()
            out["dv"] = norm_back(dp if a["post_w"] is None else dp * Num(a["post_w"]), vn, vr, a["post"])
    return out


def half_unit(dt):
    return 2.0 ** -8 if dt == BF16 else 2.0 ** -24


def check(name, got, want, dt=F32):
    got = got.float().cpu().numpy().astype(np.float64)
    slack = UNITS * want.m
    bound = slack + half_unit(dt) * (np.abs(want.v) + slack) + 1e-38
    off = np.abs(got - want.v)
    assert np.isfinite(got).all() and (off <= bound).all(), "%s: %.3g over the bound %.3g" % (name, (off - bound).max(), bound.flat[(off - bound).argmax()])


def to_dev(torch, a, dt, shift=0):
    """Device tensor of the values (rounded to the type), starting `shift` elements behind an aligned address, and the values."""
    if a is None:
        return None, None
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16 if dt == BF16 else torch.float32)
    store = torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")
    d = store[shift:shift + t.numel()].view(t.shape)
    d.copy_(t)
    return d, t.float().cpu().numpy().astype(np.float64)


def make(T, d, seed, post=RMS, nxt=RMS, gate="channel", bias=True, weights=True, alpha=0.75, with_v=True, dy=True, du=True):
    r = np.random.default_rng(seed)
    vec = lambda: 1.0 + 0.3 * r.standard_normal(d)     # noqa: E731
    a = dict(h=2.0 * r.standard_normal((T, d)) + 0.3, v=1.5 * r.standard_normal((T, d)) - 0.2 if with_v else None, post=post if with_v else NONE,
             next=nxt, alpha=np.float32(alpha).item(), dy=r.standard_normal((T, d)) if dy else None,
             du=r.standard_normal((T, d)) if du and nxt != NONE else None)
    p, n = with_v and post != NONE, nxt != NONE
    a["post_w"], a["post_b"] = (vec() if p and weights else None), (0.3 * r.standard_normal(d) if p and bias else None)
    a["next_w"], a["next_b"] = (vec() if n and weights else None), (0.3 * r.standard_normal(d) if n and bias else None)
    a["gate"] = None if gate == "none" or not with_v else 0.5 + 0.3 * r.standard_normal((1 if gate == "channel" else T, d))
    return a


TYPES = {"h": "h", "y": "h", "dy": "h", "dh": "h", "v": "v", "dv": "v", "u": "u", "du": "u"}


def run(torch, B, a, dts=(BF16, BF16, BF16), shift=0, back=True, stream=None):
    """Calls the library on the inputs of `a` (types of v, h, u); returns the outputs and the values the inputs were rounded to."""
    dt = dict(zip("vhu", dts))
    T, d = a["h"].shape
    dev, val = {}, dict(a)
    for n in ("h", "v", "dy", "du", "post_w", "post_b", "next_w", "next_b", "gate"):
        dev[n], val[n] = to_dev(torch, a[n], dt[TYPES[n]] if n in TYPES else F32, shift)
    new = lambda n, shape=(T, d): to_dev(torch, np.full(shape, np.nan), dt[TYPES[n]] if n in TYPES else F32, shift)[0]   # noqa: E731
    out, need = {}, a["dy"] is not None or a["du"] is not None
    ws = torch.full((max(B.moe_workspace_bytes(B.MOE_OP_BLOCK_END_BACKWARD, T, d, 0, 0, 0, 0), 16) // 4,), float("nan"), device="cuda")
    stats = torch.full((T, 4 if a["v"] is not None else 2), float("nan"), device="cuda")
    if a["next"] != NONE:
        out["u"] = new("u")
    torch.cuda.synchronize()
    if a["v"] is None:
        B.moe_norm(dev["h"], dt["h"], dev["next_w"], dev["next_b"], T, d, a["next"], EPS, out["u"], dt["u"], stats, stream)
        if back and need:
            out["dh"] = new("dh")
            for n in ("dnext_w", "dnext_b"):
                out[n] = new(n, (d,))
            B.moe_norm_backward(dev["du"], dt["u"], dev["h"], dt["h"], dev["next_w"], stats, T, d, a["next"], dev["dy"], out["dh"], out["dnext_w"],
                                out["dnext_b"], ws, ws.numel() * 4, stream)
    else:
        rows = 0 if a["gate"] is None else a["gate"].shape[0]
        out["y"] = new("y")
        B.moe_block_end(dev["v"], dt["v"], dev["h"], dt["h"], T, d, a["post"], EPS, dev["post_w"], dev["post_b"], dev["gate"], rows, a["alpha"],
                        a["next"], EPS, dev["next_w"], dev["next_b"], out["y"], out.get("u"), dt["u"], stats, stream)
        if back and need:
            out["dv"], out["dh"] = new("dv"), new("dh")
            if a["gate"] is not None:
                out["dgate"] = new("dgate", (rows, d))
            if a["post"] != NONE:
                out["dpost_w"], out["dpost_b"] = new("dpost_w", (d,)), new("dpost_b", (d,))
            if a["du"] is not None:
                out["dnext_w"], out["dnext_b"] = new("dnext_w", (d,)), new("dnext_b", (d,))
            B.moe_block_end_backward(dev["dy"], dev["du"], dt["u"], dev["v"], dt["v"], dev["h"], dt["h"], T, d, a["post"], dev["post_w"],
                                     dev["post_b"], dev["gate"], rows, a["alpha"], a["next"], dev["next_w"], stats, out["dv"], out["dh"],
                                     out.get("dpost_w"), out.get("dpost_b"), out.get("dgate"), out.get("dnext_w"), out.get("dnext_b"), ws,
                                     ws.numel() * 4, stream)
    torch.cuda.synchronize()
    return out, val, dt


def compare(out, val, dt):
    ref = reference(val)
    assert sorted(out) == sorted(n for n in ref if n in out) and set(out) >= {"y", "u", "dv", "dh"} & set(ref)
    for n, t in out.items():
        check(n, t, ref[n], dt[TYPES[n]] if n in TYPES else F32)


@pytest.mark.parametrize("T,d", [(1, 1), (1, 8), (3, 7), (5, 64), (2, 65), (9, 512), (3, 513), (257, 777), (33, 1032), (1, 2048), (5, 4095), (7, 4096),
                                 (3, 4104), (2, 8192), (3000, 520)])
@pytest.mark.parametrize("kind", [RMS, LAYER])
def test_norm_and_its_gradients(T, d, kind):
    torch, B = _torch()
    print("[case] norm", T, d, kind, flush=True)
    a = make(T, d, 10 * T + d + kind, nxt=kind, with_v=False)
    compare(*run(torch, B, a))
    compare(*run(torch, B, dict(a, dy=None, next_b=None), (F32, F32, F32)))


@pytest.mark.parametrize("T,d", [(1, 16), (4, 7), (6, 512), (3, 520), (129, 777), (40, 2048), (5, 4096), (3, 4104), (2, 8192), (1100, 768)])
@pytest.mark.parametrize("post,nxt,gate", [(RMS, RMS, "channel"), (LAYER, LAYER, "token"), (NONE, RMS, "none"), (RMS, NONE, "channel"),
                                           (NONE, NONE, "token"), (LAYER, RMS, "none")])
def test_block_end_and_its_gradients(T, d, post, nxt, gate):
    torch, B = _torch()
    print("[case] block end", T, d, post, nxt, gate, flush=True)
    a = make(T, d, T + 3 * d + 7 * post + nxt, post, nxt, gate)
    compare(*run(torch, B, a))
    compare(*run(torch, B, dict(a, post_b=None, next_b=None), (F32, F32, F32)))


# More rows than a launch has work-groups (wavefronts, up to 512 columns) for, and no multiple of them: the second and later rows of one, whose
# loads are under way while the row before is worked on, whose sums take the LDS buffers in turn and whose parameters' gradients are added to
# those of the rows before.  Rows in work: 8192 up to 512 columns, 2048 up to 2048, 512 up to 8192 forward; 1024 at most backward.
MANY = [(9001, 256), (4500, 777), (2500, 2048), (1100, 4104), (1100, 8192)]


@pytest.mark.parametrize("T,d", MANY)
@pytest.mark.parametrize("kind,dt", [(RMS, BF16), (LAYER, F32)])
def test_norm_of_many_rows(T, d, kind, dt):
    torch, B = _torch()
    print("[case] norm of many rows", T, d, kind, dt, flush=True)
    compare(*run(torch, B, make(T, d, T + d, nxt=kind, with_v=False), (dt, dt, dt)))


@pytest.mark.parametrize("T,d", [(8700, 136), (2500, 1032), (1300, 4096), (1100, 4104), (600, 8192)])
@pytest.mark.parametrize("post,nxt,gate,dt", [(RMS, LAYER, "token", BF16), (LAYER, RMS, "token", F32), (RMS, RMS, "channel", BF16)])
def test_block_end_of_many_rows(T, d, post, nxt, gate, dt):
    torch, B = _torch()
    print("[case] block end of many rows", T, d, post, nxt, gate, dt, flush=True)
    compare(*run(torch, B, make(T, d, T + d, post, nxt, gate), (dt, dt, dt)))


@pytest.mark.parametrize("T,d,k", [(8200, 264, 3), (2500, 2048, 2), (1300, 4096, 4), (1000, 4104, 2), (700, 8192, 5)])
def test_rows_form_of_many_rows(T, d, k):
    """The rows form, bit for bit against combine and block end, which are compared with the formula above."""
    torch, B = _torch()
    print("[case] rows form of many rows", T, d, k, flush=True)
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *shape: torch.empty(shape, device="cuda").normal_(generator=g)     # noqa: E731
    rows, shared, h, gate = new(T * k, d), new(T, d), new(T, d).bfloat16(), new(T, d)
    inv, gw = torch.randperm(T * k, generator=g, device="cuda").int(), new(T, k)
    par = [new(d) for _ in range(4)]
    norms = (LAYER, EPS, par[0], par[1], gate, T, 0.75, RMS, EPS, par[2], par[3])
    v = torch.empty((T, d), device="cuda")
    y, u, y2, u2 = (torch.full((T, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    torch.cuda.synchronize()
    B.moe_block_end_rows(rows, inv, gw, shared, k, h, BF16, T, d, *norms, y, u, BF16)
    B.moe_unpermute_combine(rows, inv, gw, shared, T, d, k, v)
    B.moe_block_end(v, F32, h, BF16, T, d, *norms, y2, u2, BF16)
    torch.cuda.synchronize()
    assert torch.isfinite(y).all() and torch.isfinite(u).all() and torch.equal(y, y2) and torch.equal(u, u2)


def test_rows_beyond_what_32_bits_reach():
    """Tensors of more than 2^31 values and 4 GiB: the last rows' bits, and those of the first, are those of a call on these rows alone."""
    torch, B = _torch()
    T, d, n = 1 << 20, 2056, 5
    print("[case] long tensors", T, d, flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *shape, dt=torch.bfloat16: torch.empty(shape, dtype=dt, device="cuda").normal_(generator=g)    # noqa: E731
    w, b = new(d, dt=torch.float32), new(d, dt=torch.float32)
    ws = torch.empty(B.moe_workspace_bytes(B.MOE_OP_NORM_BACKWARD, T, d, 0, 0, 0, 0), dtype=torch.uint8, device="cuda")
    x, du = new(T, d), new(T, d)
    assert x.numel() > 2 ** 31 and x.numel() * 2 > 2 ** 32

    def norms(x, du):
        t = x.shape[0]
        u, dx, stats, db = torch.empty_like(x), torch.empty_like(x), torch.empty((t, 2), device="cuda"), torch.empty(d, device="cuda")
        B.moe_norm(x, BF16, w, b, t, d, LAYER, EPS, u, BF16, stats)
        B.moe_norm_backward(du, BF16, x, BF16, w, stats, t, d, LAYER, du, dx, None, db, ws, ws.numel())
        torch.cuda.synchronize()
        return u, dx, stats, db

    whole = norms(x, du)
    for part in (slice(0, n), slice(T - n, T)):
        alone = norms(x[part].clone(), du[part].clone())
        assert all(torch.equal(a[part], p) for a, p in zip(whole[:3], alone[:3]))
    # (a thread adds up T / 1024 rows, then 64 + 16 parts follow: as many roundings in a row)
    total = sum(du[i:i + 65536].double().sum(0) for i in range(0, T, 65536))
    size = sum(du[i:i + 65536].double().abs().sum(0) for i in range(0, T, 65536))
    assert ((whole[3].double() - total).abs() <= (T // 1024 + 80) * 2.0 ** -24 * size).all()
    del whole, du
    # the rows form: experts' rows of 8 GiB, those of the last tokens anywhere in them
    k, tokens = 2, T // 2
    rows, inv = new(T, d, dt=torch.float32), torch.randperm(T, generator=g, device="cuda").int()
    inv[-2 * n:] = torch.arange(T - 2 * n, T, device="cuda").int()
    gw, h = new(tokens, k, dt=torch.float32), x[:tokens]

    def ends(inv, gw, h, shared):
        t = h.shape[0]
        y, u = torch.empty_like(h), torch.empty_like(h)
        B.moe_block_end_rows(rows, inv, gw, shared, k, h, BF16, t, d, RMS, EPS, w, None, None, 0, 0.5, LAYER, EPS, w, b, y, u, BF16)
        torch.cuda.synchronize()
        return y, u

    shared = new(tokens, d, dt=torch.float32)
    whole = ends(inv, gw, h, shared)
    for part in (slice(0, n), slice(tokens - n, tokens)):
        alone = ends(inv[part.start * k:part.stop * k].clone(), gw[part].clone(), h[part].clone(), shared[part].clone())
        assert all(torch.equal(a[part], p) and torch.isfinite(p).all() for a, p in zip(whole, alone))


def test_many_rows_do_not_touch_one_another():
    """A row of NaN, of infinities or of zeros between others that the same work-group goes over leaves these alone."""
    torch, B = _torch()
    for T, d in ((9001, 128), (1100, 4104)):
        a = make(T, d, 77, LAYER, RMS, "token", dy=False, du=False)
        base, _, _ = run(torch, B, a)
        bad = dict(a, h=a["h"].copy(), v=a["v"].copy())
        hit = np.arange(3, T, 7)
        bad["h"][hit[0::3]], bad["v"][hit[1::3]], bad["v"][hit[2::3], d - 1] = np.nan, 0.0, np.inf
        got, _, _ = run(torch, B, bad)
        keep = torch.ones(T, dtype=torch.bool)
        keep[torch.from_numpy(hit)] = False
        keep = keep.cuda()
        for n in ("y", "u"):
            assert torch.equal(base[n][keep], got[n][keep]), n
            assert got[n][torch.from_numpy(hit[0::3]).cuda()].isnan().all() and torch.isfinite(got[n][torch.from_numpy(hit[1::3]).cuda()]).all()


@pytest.mark.parametrize("dts", [(v, h, u) for v in (F32, BF16) for h in (F32, BF16) for u in (F32, BF16)])
@pytest.mark.parametrize("d,shift", [(264, 0), (264, 1), (8192, 0), (101, 3)])
def test_types_alignment_and_missing_parameters(dts, d, shift):
    torch, B = _torch()
    print("[case] types", dts, d, shift, flush=True)
    compare(*run(torch, B, make(5, d, d + shift, LAYER, RMS, "channel", bias=False, weights=False), dts, shift))
    compare(*run(torch, B, make(5, d, d + shift, with_v=False), dts, shift))


@pytest.mark.parametrize("only", ["dy", "du"])
def test_one_of_the_two_gradients(only):
    torch, B = _torch()
    a = make(17, 384, 5)
    compare(*run(torch, B, dict(a, dy=a["dy"] if only == "dy" else None, du=a["du"] if only == "du" else None)))


@pytest.mark.parametrize("k", [1, 2, 3, 4, 5, 8, 11])
@pytest.mark.parametrize("T,d,shared", [(1, 64, True), (37, 520, False), (19, 777, True), (3, 4104, True), (300, 2048, False)])
def test_rows_form_is_combine_and_block_end(k, T, d, shared):
    """The experts' rows, weighted and summed on the way: the bits of moe_unpermute_combine followed by moe_block_end (of the
    formula where the width is not one that moe_unpermute_combine takes)."""
    torch, B = _torch()
    print("[case] rows", k, T, d, shared, flush=True)
    r = np.random.default_rng(k + T)
    a = make(T, d, k, LAYER if k % 2 else NONE, RMS, "channel", dy=False, du=False)
    A = T * k
    rows, inv = r.standard_normal((A, d)).astype(np.float32), r.permutation(A).astype(np.int32)
    gw, sh = r.random((T, k)).astype(np.float32), r.standard_normal((T, d)).astype(np.float32) if shared else None
    cu = lambda x: None if x is None else torch.from_numpy(x).cuda()    # noqa: E731
    rows_d, inv_d, gw_d, sh_d = cu(rows), cu(inv), cu(gw), cu(sh)
    dev = {n: to_dev(torch, a[n], BF16 if n == "h" else F32)[0] for n in ("h", "post_w", "post_b", "next_w", "next_b", "gate")}
    y, u, y2, u2 = (torch.empty((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    norms = (a["post"], EPS, dev["post_w"], dev["post_b"], dev["gate"], 1, a["alpha"], a["next"], EPS, dev["next_w"], dev["next_b"])
    B.moe_block_end_rows(rows_d, inv_d, gw_d, sh_d, k, dev["h"], BF16, T, d, *norms, y, u, BF16)
    v = np.einsum("tk,tkd->td", gw.astype(np.float64), rows.astype(np.float64)[inv].reshape(T, k, d)) + (0 if sh is None else sh)
    if d % 4 == 0:
        v_d = torch.empty((T, d), device="cuda")
        B.moe_unpermute_combine(rows_d, inv_d, gw_d, sh_d, T, d, k, v_d)
        B.moe_block_end(v_d, F32, dev["h"], BF16, T, d, *norms, y2, u2, BF16)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(u, u2)
    torch.cuda.synchronize()
    ref = reference(dict(a, v=v, h=dev["h"].float().cpu().numpy().astype(np.float64), **{
        n: dev[n].cpu().numpy().astype(np.float64) for n in ("post_w", "post_b", "next_w", "next_b", "gate") if dev[n] is not None}))
    check("y", y, ref["y"], BF16)
    check("u", u, ref["u"], BF16)


def test_rows_form_missing_rows():
    """An assignment without a row adds nothing at weight zero, makes its token NaN otherwise and touches no other token."""
    torch, B = _torch()
    T, d, k = 5, 136, 2
    r = np.random.default_rng(3)
    rows, h = torch.from_numpy(r.standard_normal((T * k, d)).astype(np.float32)).cuda(), torch.from_numpy(r.standard_normal((T, d)).astype(np.float32)).cuda()
    inv, gw = torch.arange(T * k, dtype=torch.int32).cuda(), torch.full((T, k), 0.5).cuda()
    y, u = torch.empty((T, d), device="cuda"), torch.empty((T, d), device="cuda")

    def call(inv, gw):
        B.moe_block_end_rows(rows, inv, gw, None, k, h, F32, T, d, NONE, 0.0, None, None, None, 0, 1.0, RMS, EPS, None, None, y, u, F32)
        torch.cuda.synchronize()
        return y.clone(), u.clone()

    y0, u0 = call(inv, gw)
    inv[3] = -1                                        # token 1, second choice
    y1, u1 = call(inv, gw)
    keep = torch.tensor([0, 2, 3, 4]).cuda()
    assert y1[1].isnan().all() and u1[1].isnan().all() and torch.equal(y0[keep], y1[keep]) and torch.equal(u0[keep], u1[keep])
    gw[1, 1] = 0.0
    y2, _ = call(inv, gw)
    assert torch.equal(y2[1], h[1] + 0.5 * rows[2]) and torch.equal(y0[keep], y2[keep])


def _loss(a):
    """sum dy y + sum du u in 64 bits, plainly."""
    def n(x, kind):
        if kind == LAYER:
            x = x - x.mean(1, keepdims=True)
        return x / np.sqrt((x * x).mean(1, keepdims=True) + EPS)
    p = a["v"] if a["post"] == NONE else n(a["v"], a["post"]) * a["post_w"] + a["post_b"]
    y = a["alpha"] * a["h"] + a["gate"] * p
    return (a["dy"] * y).sum() + (a["du"] * (n(y, a["next"]) * a["next_w"] + a["next_b"])).sum()


@pytest.mark.parametrize("post,nxt,gate", [(RMS, LAYER, "channel"), (LAYER, RMS, "token")])
def test_gradients_against_differences(post, nxt, gate):
    """Central differences of the loss in 64 bits, step 1e-4: their own error is of the order of step^2 times third derivatives
    of order one; the kernels work in fp32 on sums of at most 3 x 24 terms of order one."""
    torch, B = _torch()
    a = make(3, 24, 11, post, nxt, gate)
    out, val, _ = run(torch, B, a, (F32, F32, F32))
    for name, grad in (("h", "dh"), ("v", "dv"), ("post_w", "dpost_w"), ("post_b", "dpost_b"), ("next_w", "dnext_w"), ("next_b", "dnext_b"), ("gate", "dgate")):
        got = out[grad].cpu().numpy().astype(np.float64)
        for at in list(np.ndindex(got.shape))[::5]:
            up, down = dict(val, **{name: val[name].copy()}), dict(val, **{name: val[name].copy()})
            up[name][at] += 1e-4
            down[name][at] -= 1e-4
            slope = (_loss(up) - _loss(down)) / 2e-4
            assert abs(slope - got[at]) <= 2e-5 * (1 + abs(slope)), (grad, at, slope, got[at])


@pytest.mark.parametrize("kind", [RMS, LAYER])
@pytest.mark.parametrize("d", [48, 777, 2048, 8192])
def test_rows_do_not_touch_one_another(kind, d):
    """Zero rows, infinities and NaN stay in their row."""
    torch, B = _torch()
    a = make(6, d, 21, kind, kind, "channel", dy=False, du=False)
    base, _, _ = run(torch, B, a)
    bad = dict(a, h=a["h"].copy(), v=a["v"].copy())
    bad["h"][1], bad["v"][1] = 0.0, 0.0
    bad["h"][2, d // 2], bad["v"][4, 0] = np.inf, np.nan
    got, val, dt = run(torch, B, bad)
    for n in ("y", "u"):
        for t in (0, 3, 5):
            assert torch.equal(base[n][t], got[n][t])
        assert got[n][4].isnan().any()
    assert got["u"][2].isnan().any()
    ref = reference({n: v[1:2] if isinstance(v, np.ndarray) and v.shape[:1] == (6,) else v for n, v in val.items()})
    check("y of zeros", got["y"][1:2], ref["y"], BF16)
    check("u of zeros", got["u"][1:2], ref["u"], BF16)


def test_in_place_and_twice_the_same_bits():
    torch, B = _torch()
    T, d = 700, 1024
    a = make(T, d, 31)
    out, val, _ = run(torch, B, a)
    again, _, _ = run(torch, B, a)
    assert all(torch.equal(out[n], again[n]) for n in out)
    dev = {n: to_dev(torch, a[n], BF16 if n in TYPES else F32)[0] for n in ("h", "v", "dy", "du", "post_w", "post_b", "next_w", "next_b", "gate")}
    ws = torch.empty(B.moe_workspace_bytes(B.MOE_OP_BLOCK_END_BACKWARD, T, d, 0, 0, 0, 0), dtype=torch.uint8, device="cuda")
    stats, u = torch.empty((T, 4), device="cuda"), torch.empty_like(dev["h"])
    y = dev["h"].clone()
    B.moe_block_end(dev["v"], BF16, y, BF16, T, d, RMS, EPS, dev["post_w"], dev["post_b"], dev["gate"], 1, a["alpha"], RMS, EPS, dev["next_w"],
                    dev["next_b"], y, u, BF16, stats)
    dv, dh = dev["v"].clone(), dev["dy"].clone()
    B.moe_block_end_backward(dh, dev["du"], BF16, dv, BF16, dev["h"], BF16, T, d, RMS, dev["post_w"], dev["post_b"], dev["gate"], 1, a["alpha"], RMS,
                             dev["next_w"], stats, dv, dh, None, None, None, None, None, None, 0)
    torch.cuda.synchronize()
    assert torch.equal(y, out["y"]) and torch.equal(u, out["u"]) and torch.equal(dv, out["dv"]) and torch.equal(dh, out["dh"])


def test_no_rows():
    """No tokens: outputs stay alone, the parameters' gradients are zero."""
    torch, B = _torch()
    d = 520
    dw, db, dg = (torch.full((d,), 7.0, device="cuda") for _ in range(3))
    B.moe_norm(None, BF16, None, None, 0, d, RMS, EPS, None, BF16)
    B.moe_norm_backward(None, BF16, None, BF16, None, None, 0, d, RMS, None, None, dw, db, None, 0)
    gate = torch.ones(d, device="cuda")
    B.moe_block_end_backward(None, None, BF16, None, BF16, None, BF16, 0, d, NONE, None, None, gate, 1, 1.0, NONE, None, None, None, None, None, None,
                             dg, None, None, None, 0)
    torch.cuda.synchronize()
    assert not dw.any() and not db.any() and not dg.any()


def test_no_rows_of_a_token_gate():
    """No tokens and a gate for every token: dgate has no rows, and what lies at its address stays; the others are zero."""
    torch, B = _torch()
    d = 264
    dpw, dpb, other = (torch.full((d,), 7.0, device="cuda") for _ in range(3))
    B.moe_block_end_backward(None, None, BF16, None, BF16, None, BF16, 0, d, RMS, None, None, torch.ones(d, device="cuda"), 0, 1.0, NONE, None, None, None,
                             None, dpw, dpb, other, None, None, None, 0)
    torch.cuda.synchronize()
    assert not dpw.any() and not dpb.any() and (other == 7.0).all()


def test_stream_and_graph():
    """The calls go to the stream that they are given, and a graph of them replays on new inputs."""
    torch, B = _torch()
    T, d = 65, 1536
    a, b = make(T, d, 41, with_v=False), make(T, d, 42, with_v=False)
    side = torch.cuda.Stream()
    out, val, dt = run(torch, B, a, stream=side)
    compare(out, val, dt)
    x, w, u = to_dev(torch, a["h"], BF16)[0], to_dev(torch, a["next_w"], F32)[0], torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    du, dx = to_dev(torch, a["du"], BF16)[0], torch.empty_like(u)
    stats, dw = torch.empty((T, 2), device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(B.moe_workspace_bytes(B.MOE_OP_NORM_BACKWARD, T, d, 0, 0, 0, 0), dtype=torch.uint8, device="cuda")

    def calls():
        B.moe_norm(x, BF16, w, None, T, d, RMS, EPS, u, BF16, stats)
        B.moe_norm_backward(du, BF16, x, BF16, w, stats, T, d, RMS, None, dx, dw, None, ws, ws.numel())

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for src in (b, a, b):
        x.copy_(to_dev(torch, src["h"], BF16)[0])
        calls()
        torch.cuda.synchronize()
        want = [t.clone() for t in (u, dx, dw)]
        for t in (u, dx, dw):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, (u, dx, dw)))
