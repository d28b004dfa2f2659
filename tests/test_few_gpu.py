"""moe_layer_few against the layer's definition in 64 bits (plain numpy, here), over token counts from 1 to the limit, odd numbers of
experts, ragged widths, both activations, shared experts, both types; the choice bit-exact.

Tolerance.  fp32: a chain of at most d + F roundings would allow (d + F) 2^-24 of the sums of absolute values; partial
sums of at most 16 x 32 terms in a row, then 16 wavefronts: 600 units of 2^-24 of the output's magnitude, computed
beside the reference with the magnitudes of both products.  bf16: the hidden activations are rounded to 11 bits (2^-12 relative) before the second
product, and a bf16 output to 8 bits (2^-8 of itself at most)."""
import numpy as np
import pytest

import moe_workloads as W

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    from paper_2506_12417_amd import binding as B
    from paper_2506_12417_amd.layer import ExpertGroup, to_device
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return torch, B, ExpertGroup, to_device


def rounded(a, dt):
    return W.f32_to_bf16_bits(a.astype(np.float32)) if dt == "bf16" else a.astype(np.float32)


def wide(a):
    return W.bf16_bits_to_f32(a).astype(np.float64) if a.dtype == np.uint16 else a.astype(np.float64)


class Case:
    def __init__(self, T, d, F, E, k, act, dt, shared_F=0, renorm=0, seed=0, bias=True, x=None, W_g=None, b=None):
        r = np.random.default_rng([seed, T, d, F, E, k])
        self.T, self.d, self.F, self.E, self.k, self.act, self.dt, self.shared_F, self.renorm = T, d, F, E, k, act, dt, shared_F, renorm
        self.x = rounded(r.standard_normal((T, d)) if x is None else x, dt)
        self.W_g = rounded(r.standard_normal((d, E)) / np.sqrt(d) if W_g is None else W_g, dt)
        self.b = b if b is not None else (0.5 * r.standard_normal(E)).astype(np.float32) if bias else None
        mk = lambda n, i, o: rounded(r.standard_normal((n, i, o)) / np.sqrt(i), dt)    # noqa: E731
        self.w = dict(W1=mk(E, d, F), W2=mk(E, F, d)) if act == "relu" else dict(Wg=mk(E, d, F), Wu=mk(E, d, F), Wd=mk(E, F, d))
        self.sw = dict(Wg=mk(1, d, shared_F), Wu=mk(1, d, shared_F), Wd=mk(1, shared_F, d)) if shared_F else None


def ffn(x, w, e, sat):
    """Output and magnitude (for the error bound) of rows x."""
    if "W1" in w:
        w1, w2 = wide(w["W1"][e]), wide(w["W2"][e])
        h, hm = np.maximum(x @ w1, 0.0), np.abs(x) @ np.abs(w1)
    else:
        wg, wu, w2 = wide(w["Wg"][e]), wide(w["Wu"][e]), wide(w["Wd"][e])
        g, u = x @ wg, x @ wu
        with np.errstate(over="ignore"):
            s = g / (1.0 + np.exp(-g))
        h, hm = s * u, 1.1 * (np.abs(x) @ np.abs(wg)) * np.abs(u) + np.abs(s) * (np.abs(x) @ np.abs(wu))
    if sat:
        h = np.clip(h, -65504.0, 65504.0)
    return h @ w2, hm @ np.abs(w2), np.abs(h) @ np.abs(w2)


def reference(c):
    x = wide(c.x)
    logits = x @ wide(c.W_g) + (0.0 if c.b is None else c.b.astype(np.float64))
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :c.k]
    e = np.exp(logits - logits.max(1, keepdims=True))
    gate = np.take_along_axis(e / e.sum(1, keepdims=True), idx, 1)
    if c.renorm:
        gate = gate / gate.sum(1, keepdims=True)
    y, m1, m2 = np.zeros((3, c.T, c.d))
    for ex in np.unique(idx):
        t, j = np.nonzero(idx == ex)
        for into, part in zip((y, m1, m2), ffn(x[t], c.w, ex, c.dt == "bf16")):
            into[t] += part * gate[t, j][:, None]
    if c.sw:
        for into, part in zip((y, m1, m2), ffn(x, c.sw, 0, c.dt == "bf16")):
            into += part
    return idx, gate, y, m1, m2


class Device:
    """The case's parameters as the library takes them."""

    def __init__(self, c):
        self.torch, self.B, Group, to_dev = _torch()
        B, torch = self.B, self.torch
        dev = torch.device("cuda:0")
        self.dt = B.MOE_BF16 if c.dt == "bf16" else B.MOE_F32
        self.act = B.MOE_SWIGLU if c.act == "swiglu" else B.MOE_RELU
        self.x, self.W_g = to_dev(c.x, dev), to_dev(c.W_g, dev)
        self.b = None if c.b is None else to_dev(c.b, dev)
        self.norm2, self.W = None, self.W_g
        if c.dt == "bf16":
            self.W, self.norm2 = torch.empty((c.E, c.d), dtype=torch.bfloat16, device=dev), torch.empty(c.E, device=dev)
            B.moe_pack_router(self.W_g, c.d, c.E, self.dt, self.W, self.norm2)
        self.g = Group(c.E, c.d, c.F, self.act, self.dt, dev)
        for e in range(c.E):
            self.g.load_expert(e, {n: a[e] for n, a in c.w.items()})
        self.s = None
        if c.sw:
            self.s = Group(1, c.d, c.shared_F, B.MOE_SWIGLU, self.dt, dev)
            self.s.load_expert(0, {n: a[0] for n, a in c.sw.items()})
        self.idx = torch.full((c.T, c.k), -7, dtype=torch.int32, device=dev)
        self.gate = torch.full((c.T, c.k), float("nan"), device=dev)
        n = B.moe_layer_few_workspace(c.T, c.F, c.k, c.shared_F, self.dt)
        self.ws = torch.full((max(n, 16) // 2,), float("nan"), dtype=torch.float16, device=dev)
        self.c = c

    def run(self, y_dt=None, x=None, stream=None):
        c, B, torch = self.c, self.B, self.torch
        y_dt = B.MOE_F32 if y_dt is None else y_dt
        y = torch.full((c.T, c.d), float("nan"), dtype=torch.float32 if y_dt == B.MOE_F32 else torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        B.moe_layer_few(self.x if x is None else x, c.T, c.d, c.F, c.E, c.k, self.act, self.dt, c.renorm, self.W, self.norm2, self.b, self.g.in_ptrs,
                        self.g.out_ptrs, c.shared_F, self.s.in_ptrs if self.s else None, self.s.out_ptrs if self.s else None, self.idx, self.gate,
                        self.ws, self.ws.numel() * 2, y, y_dt, stream)
        torch.cuda.synchronize()
        return y


def check(c, y_dts=(0, 1)):
    dev = Device(c)
    idx, gate, y, m1, m2 = reference(c)
    for y_dt in y_dts:
        got = dev.run(y_dt).float().cpu().numpy()
        assert np.array_equal(dev.idx.cpu().numpy(), idx), "expert indices differ"
        assert np.abs(dev.gate.cpu().numpy() - gate).max() <= 2e-6
        # (a gate's own error is 2e-6 of the terms it weights)
        bound = 600 * 2.0 ** -24 * m1 + (600 * 2.0 ** -24 + 4e-6) * m2 + (2.0 ** -12 * m2 if c.dt == "bf16" else 0.0)
        bound += 2.0 ** -8 * (np.abs(y) + bound) if y_dt else 0.0
        off = np.abs(got - y) - bound
        assert np.isfinite(got).all() and (off <= 0).all(), "%.3g over the bound" % off.max()


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 48, 49, 64])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_token_counts(T, dt):
    print("[case] few T=%d %s" % (T, dt), flush=True)
    check(Case(T, 192, 320, 5, 2, "swiglu", dt, shared_F=128, renorm=T % 2))


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (7, 1), (8, 8), (15, 3), (16, 4), (17, 2), (60, 4), (64, 6), (65, 8), (128, 1), (129, 5), (256, 8)])
@pytest.mark.parametrize("dt,act,T", [("bf16", "relu", 5), ("bf16", "swiglu", 50), ("f32", "relu", 11)])
def test_experts_and_choices(E, k, dt, act, T):
    print("[case] few E=%d k=%d %s %s T=%d" % (E, k, dt, act, T), flush=True)
    check(Case(T, 128, 64, E, k, act, dt, renorm=k % 2, bias=E % 2 == 0), y_dts=(0,))


@pytest.mark.parametrize("T,d,E,k,shared_F", [(5, 256, 160, 4, 0), (16, 2048, 144, 2, 0), (16, 2048, 160, 2, 2048), (20, 256, 80, 3, 0), (31, 1024, 90, 2, 0),
                                              (32, 960, 200, 4, 64), (40, 256, 160, 2, 0), (64, 4096, 150, 1, 0)])
def test_wavefronts_without_experts(T, d, E, k, shared_F):
    """Numbers of experts that leave wavefronts of the routing none: these copy their rows of x into LDS like the others, and
    those rows have to be there before anybody reads them (beside the first product, too, and in a launch of its own)."""
    print("[case] few idle wavefronts T=%d d=%d E=%d k=%d shared=%d" % (T, d, E, k, shared_F), flush=True)
    check(Case(T, d, 64, E, k, "relu", "bf16", shared_F=shared_F, renorm=1), y_dts=(0,))


@pytest.mark.parametrize("d,F,shared_F", [(64, 64, 0), (64, 128, 64), (320, 1984, 0), (768, 512, 192), (1088, 704, 0), (4096, 64, 64), (4160, 128, 0), (8192, 192, 0)])
@pytest.mark.parametrize("dt,act,T", [("bf16", "swiglu", 3), ("bf16", "relu", 21), ("f32", "swiglu", 9)])
def test_widths(d, F, shared_F, dt, act, T):
    print("[case] few d=%d F=%d shared=%d %s %s" % (d, F, shared_F, dt, act), flush=True)
    check(Case(T, d, F, 4, 2, act, dt, shared_F=shared_F, renorm=1), y_dts=(1,))


@pytest.mark.parametrize("T,d,F,E,k,shared_F", [(5, 320, 512, 24, 4, 0), (12, 64, 128, 9, 3, 64), (20, 256, 192, 16, 8, 128), (23, 768, 256, 6, 2, 0),
                                                (33, 640, 320, 12, 3, 64), (47, 512, 448, 24, 6, 0), (64, 960, 1472, 8, 2, 0), (64, 64, 64, 3, 1, 64)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_narrow_layers(T, d, F, E, k, shared_F, dt):
    """Few output columns and many tokens: those who share the columns take ranges of the tokens, of odd lengths here."""
    print("[case] few narrow T=%d d=%d F=%d E=%d k=%d shared=%d %s" % (T, d, F, E, k, shared_F, dt), flush=True)
    check(Case(T, d, F, E, k, "swiglu" if T % 2 else "relu", dt, shared_F=shared_F, renorm=T % 2))


@pytest.mark.parametrize("T,d,F,E,k,shared_F", [(1, 2048, 64, 5, 2, 2048), (9, 2048, 128, 20, 3, 2112), (16, 2048, 64, 7, 1, 2048), (16, 8192, 64, 4, 2, 512),
                                                (3, 8192, 64, 4, 2, 576), (33, 8192, 64, 4, 2, 0), (40, 4096, 64, 3, 1, 64)])
def test_large_shared_experts_and_wide_tokens(T, d, F, E, k, shared_F):
    """The shared expert's first product beside the routing, eight tokens a work-group there; tokens that do not fit LDS."""
    print("[case] few beside T=%d d=%d F=%d E=%d k=%d shared=%d" % (T, d, F, E, k, shared_F), flush=True)
    check(Case(T, d, F, E, k, "swiglu", "bf16", shared_F=shared_F, renorm=1), y_dts=(0,))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,shared_F", [(9, 0), (40, 64), (64, 0)])
def test_tokens_that_are_no_numbers_in_narrow_layers(T, shared_F, dt):
    """First, last and some in between are NaN: their rows are, no other is, and the others keep their values to the tolerance."""
    c = Case(T, 128, 192, 7, 3, "swiglu", dt, shared_F=shared_F)
    dev = Device(c)
    idx, _, y, m1, m2 = reference(c)
    x = dev.x.clone()
    bad = sorted({0, T // 2, T // 2 + 1, T - 1})
    keep = [t for t in range(T) if t not in bad]
    x[bad] = float("nan")
    got = dev.run(x=x).cpu().numpy()
    assert np.isnan(got[bad]).all() and np.array_equal(dev.idx.cpu().numpy()[keep], idx[keep])
    bound = 600 * 2.0 ** -24 * m1 + (600 * 2.0 ** -24 + 4e-6) * m2 + (2.0 ** -12 * m2 if dt == "bf16" else 0.0)
    assert (np.abs(got - y) <= bound)[keep].all()


def test_all_tokens_on_one_expert():
    """A bias that leaves one expert: 64 rows there, none elsewhere."""
    for dt in ("bf16", "f32"):
        b = np.full(9, -50.0, dtype=np.float32)
        b[4] = 50.0
        check(Case(64, 256, 192, 9, 1, "relu", dt, b=b))


def test_near_ties_are_decided_as_in_64_bits():
    """Columns of W_g that repeat others, or differ from them in one last bit: equal logits go to the lower index, and gaps far
    below what fp32 sums resolve decide."""
    r = np.random.default_rng(5)
    T, d, E = 40, 768, 24
    x = r.standard_normal((T, d))
    W_g = r.standard_normal((d, E)) / np.sqrt(d)
    W_g[:, 12:] = W_g[:, :12]                                  # every expert twice
    bits = rounded(W_g, "bf16")
    for e in range(14, 24):                                    # ten of them with one weight a bit larger or smaller
        i = int(np.abs(wide(rounded(x, "bf16"))).min(0).argmin()) + e - 14
        bits[i % d, e] ^= 1                                   # (the last bit of a weight)
    c = Case(T, d, 64, E, 4, "relu", "bf16", bias=False, x=x, W_g=wide(bits))
    logits = wide(c.x) @ wide(c.W_g)
    top = -np.sort(-logits, axis=1)[:, :5]
    assert (top[:, :-1] - top[:, 1:] < 1e-4).any(1).mean() > 0.75         # near ties nearly everywhere
    check(c, y_dts=(0,))
    c.dt = "f32"
    c.x, c.W_g, c.w = wide(c.x).astype(np.float32), wide(c.W_g).astype(np.float32), {n: wide(a).astype(np.float32) for n, a in c.w.items()}
    check(c, y_dts=(0,))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_tokens_that_are_no_numbers(dt):
    """A NaN in a token makes its own row NaN and names no expert; the other tokens' bits stay."""
    c = Case(12, 192, 128, 10, 3, "swiglu", dt, shared_F=64)
    dev = Device(c)
    y0 = dev.run()
    idx0 = dev.idx.clone()
    x = dev.x.clone()
    x[5, 17] = float("nan")
    y1 = dev.run(x=x)
    keep = [t for t in range(12) if t != 5]
    assert y1[5].isnan().all() and dev.gate[5].isnan().all() and ((dev.idx[5] < 0) | (dev.idx[5] >= c.E)).all()
    assert dev.torch.equal(y0[keep], y1[keep]) and dev.torch.equal(idx0[keep], dev.idx[keep])
    x[:] = float("nan")                                        # nobody has an expert
    assert dev.run(x=x).isnan().all()
    x = dev.x.clone()
    x[3] = 0.0                                                 # a zero token is routed by the bias alone
    y2 = dev.run(x=x)
    assert not y2[3].any() and dev.idx[3].cpu().tolist() == np.argsort(-c.b, kind="stable")[:3].tolist()


def test_masked_experts():
    """Experts masked by a bias of minus infinity, or the lowest number, are not chosen while others are left, have weight zero when
    they are, and their infinite matrices touch nobody then unless chosen."""
    for low in (-np.inf, np.finfo(np.float32).min):
        b = np.full(12, low, dtype=np.float32)
        b[[2, 7, 11]] = [0.0, 0.5, -0.25]
        check(Case(19, 128, 64, 12, 3, "relu", "bf16", b=b), y_dts=(0,))


@pytest.mark.parametrize("T,shared_F", [(5, 0), (20, 0), (40, 0), (9, 2048)])
@pytest.mark.parametrize("renorm", [0, 1])
def test_gates_keep_their_bits(T, shared_F, renorm):
    """Gates to fp32's precision relative to themselves, small ones too.  Tokens of a single one make the logits weights of W_g, so that they and
    their differences are exact.  In units of 2^-24: an exponential is off by 3 (an instruction's last place, a correction's rounding), the
    sum of positive terms by the terms' 3 and 8 additions, the quotient by 1; 3 + 3 + 8 + 1 < 16.  (A rounded product with log2(e) alone
    would be off by 2^-18 ln 2 at 2^-115, 44 units.)"""
    print("[case] few gates T=%d shared=%d renorm=%d" % (T, shared_F, renorm), flush=True)
    d, E, k = 2048 if shared_F else 128, 16, 8
    r = np.random.default_rng(T)
    x, W_g = np.zeros((T, d)), np.zeros((d, E))
    x[np.arange(T), 3 * np.arange(T)] = 1.0
    for t in range(T):
        low = -80.0 * r.random(E)
        low[r.integers(E)] = 0.0
        W_g[3 * t] = low
    c = Case(T, d, 64, E, k, "relu", "bf16", shared_F=shared_F, renorm=renorm, bias=False, x=x, W_g=W_g)
    dev = Device(c)
    dev.run()
    idx, gate, _, _, _ = reference(c)
    assert np.array_equal(dev.idx.cpu().numpy(), idx)
    off = np.abs(dev.gate.cpu().numpy().astype(np.float64) / gate - 1.0)
    assert off.max() <= 16 * 2.0 ** -24, off.max() * 2.0 ** 24


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("low", [-np.inf, float(np.finfo(np.float32).min)])
@pytest.mark.parametrize("T", [7, 29, 45])
def test_masked_experts_that_are_chosen_and_that_are_not(T, low, dt):
    """More choices than experts that are left: the masked ones follow by their index with weight zero, and the rows are those of the experts that
    are left.  As many choices as are left: the masked ones' matrices of infinities and NaN take part in nothing."""
    print("[case] few masked T=%d %g %s" % (T, low, dt), flush=True)
    E, k, left = 9, 4, [1, 6]
    b = np.full(E, low, dtype=np.float32)
    b[left] = [0.25, 0.0]
    c = Case(T, 128, 64, E, k, "relu", dt, b=b, renorm=T % 2)
    check(c, y_dts=(0,))
    dev = Device(c)
    y = dev.run()
    idx, gate = dev.idx.cpu().numpy(), dev.gate.cpu().numpy()
    assert (np.sort(idx[:, :2], 1) == left).all() and (idx[:, 2:] == [0, 2]).all() and (gate[:, 2:] == 0).all() and (gate[:, :2] > 0).all()
    for only in (1, 2):                                       # as many as are left, or fewer
        c = Case(T, 128, 64, E, only, "relu", dt, b=b, renorm=T % 2)
        dev = Device(c)
        y = dev.run()
        for e in sorted(set(range(E)) - set(left)):
            for name, w in ((n, a[e].copy()) for n, a in c.w.items()):
                w[:] = (0x7f80, 0x7fc0)[e % 2] if dt == "bf16" else (np.inf, np.nan)[e % 2]
                dev.g.load_expert(e, {n: w if n == name else a[e] for n, a in c.w.items()})
            assert dev.torch.equal(dev.run(), y), (only, e)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,F,E,k,act,shared_F", [(6, 128, 192, 5, 2, "relu", 0), (12, 768, 128, 6, 1, "relu", 0), (40, 192, 128, 7, 3, "swiglu", 64),
                                                    (30, 2048, 64, 4, 2, "swiglu", 64)])
def test_weights_that_are_no_numbers(T, d, F, E, k, act, shared_F, dt):
    """A NaN in an expert's first matrix makes the rows of the tokens that chose it NaN, one in its second matrix their outputs of that
    column, one in the shared expert's every token's; all other values keep their bits."""
    print("[case] few NaN weights T=%d d=%d %s %s" % (T, d, act, dt), flush=True)
    c = Case(T, d, F, E, k, act, dt, shared_F=shared_F)
    dev = Device(c)
    y0 = dev.run().cpu().numpy()
    idx = dev.idx.cpu().numpy()
    e = int(np.bincount(idx.ravel(), minlength=E).argmax())
    chose = (idx == e).any(1)
    nan = 0x7fc0 if dt == "bf16" else np.nan
    for name in c.w:
        w = {n: a[e].copy() for n, a in c.w.items()}
        w[name][w[name].shape[0] // 3, 17] = nan
        dev.g.load_expert(e, w)
        y = dev.run().cpu().numpy()
        want = np.zeros((T, d), dtype=bool)
        want[chose] = True
        if name in ("W2", "Wd"):
            want[:, :17] = want[:, 18:] = False
        assert np.array_equal(np.isnan(y), want) and np.array_equal(y[~want], y0[~want]), name
    dev.g.load_expert(e, {n: a[e] for n, a in c.w.items()})
    for name in c.sw or ():
        w = {n: a[0].copy() for n, a in c.sw.items()}
        w[name][0, 3] = nan
        dev.s.load_expert(0, w)
        y = dev.run().cpu().numpy()
        want = np.full((T, d), name != "Wd")
        want[:, 3] = True
        assert np.array_equal(np.isnan(y), want) and np.array_equal(y[~want], y0[~want]), name


def test_hidden_activations_saturate():
    c = Case(4, 64, 64, 2, 1, "relu", "bf16", bias=False)
    c.x = rounded(wide(c.x) * 3e4, "bf16")
    check(c, y_dts=(0,))


def test_same_bits_twice_on_a_stream_and_in_a_graph():
    c = Case(13, 768, 512, 20, 3, "swiglu", "bf16", shared_F=256)
    dev = Device(c)
    torch = dev.torch
    y0, side = dev.run(), torch.cuda.Stream()
    assert torch.equal(y0, dev.run()) and torch.equal(y0, dev.run(stream=side))
    x, y = dev.x.clone(), torch.empty_like(y0)

    def call():
        dev.B.moe_layer_few(x, c.T, c.d, c.F, c.E, c.k, dev.act, dev.dt, c.renorm, dev.W, dev.norm2, dev.b, dev.g.in_ptrs, dev.g.out_ptrs, c.shared_F,
                            dev.s.in_ptrs, dev.s.out_ptrs, dev.idx, dev.gate, dev.ws, dev.ws.numel() * 2, y, dev.B.MOE_F32)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)).to(x.dtype))
        want = dev.run(x=x)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
