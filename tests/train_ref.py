"""The training step's formulas in float64 on the host, and bounds of what rounding may change, value by value.

A rounding is off by half a step at most, relative to the value: bf16 2^-8, half 2^-11, fp32 2^-24.  A sum of n products in fp32 is off by at most
n 2^-24 times the sum of the products' magnitudes, in whatever order it is made."""
import numpy as np

U32, U16, UH = 2.0 ** -24, 2.0 ** -8, 2.0 ** -11
KEPT = 0.5 + 1e-4          # steps of its scale that a kept value may be off: half a step, and 127 / m and the product rounded in fp32


def unit(dtype):
    return U32 if dtype == "f32" else U16


def routing(T, k, E, seed, empty=(), one=None):
    """k different experts a token out of those that take part; the sort of them."""
    r = np.random.default_rng(seed)
    ids = np.array([e for e in range(E) if e not in empty])
    p = 1.0 / np.arange(1, len(ids) + 1)
    idx = np.stack([r.choice(ids, size=k, replace=False, p=p / p.sum()) for _ in range(T)]) if T else np.zeros((0, k), int)
    if one is not None:
        idx[:] = one
    return sort(idx.astype(np.int32), E)


def sort(idx, E):
    flat = idx.reshape(-1)
    on = (flat >= 0) & (flat < E)
    perm = np.array([a for a in np.argsort(np.where(on, flat, E), kind="stable") if on[a]], dtype=np.int32)
    inv = np.full(flat.size, -1, dtype=np.int32)
    inv[perm] = np.arange(perm.size)
    counts = np.bincount(flat[on], minlength=E)
    return dict(idx=idx, perm=perm, inv=inv, counts=counts, offsets=np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))


def blocks(n):
    return -(-n // 64)


def block_max(v):
    """[rows, n] -> the largest magnitude of each value's block of 64."""
    rows, n = v.shape
    p = np.zeros((rows, blocks(n) * 64))
    p[:, :n] = np.abs(v)
    return np.repeat(p.reshape(rows, -1, 64).max(2), 64, axis=1)[:, :n]


def restore(q, scale):
    return q.astype(np.float64) * np.repeat(scale.astype(np.float64), 64, axis=1)[:, :q.shape[1]]


def sigmoid(v):
    return 1.0 / (1.0 + np.exp(-v))


def first_product(x, w, rt, k, act):
    """z and the bound of its error."""
    z, err = [], []
    for e in range(len(rt["counts"])):
        rows = x[rt["perm"][rt["offsets"][e]:rt["offsets"][e + 1]] // k]
        m = np.concatenate([w[n][e] for n in "ab" if w.get(n) is not None], axis=1)
        z.append(rows @ m)
        err.append(x.shape[1] * U32 * (np.abs(rows) @ np.abs(m)))
    z, err = np.concatenate(z), np.concatenate(err)
    return (np.maximum(z, 0.0), err) if act == "relu" else (z, err)


def hidden(z, act):
    if act == "relu":
        return z
    g, u = np.split(z, 2, axis=1)
    return g * sigmoid(g) * u


def ffn_backward(x, dy, w, rt, k, gate, z, act):
    """Gradients from the kept z, each with its bound: dx_perm, dgate [A], dw a, b, o."""
    E, (d, F) = len(rt["counts"]), w["a"].shape[1:]
    A = len(rt["inv"])
    n_rows = int(rt["offsets"][-1])
    out = {n: (np.zeros_like(w[n], dtype=np.float64), np.zeros_like(w[n], dtype=np.float64)) for n in "abo" if w.get(n) is not None}
    dxp, dxe, dgate, dge = np.zeros((n_rows, d)), np.zeros((n_rows, d)), np.zeros(A), np.zeros(A)
    for e in range(E):
        sl = slice(rt["offsets"][e], rt["offsets"][e + 1])
        a = rt["perm"][sl]
        X, DY, Z = x[a // k], dy[a // k], z[sl]
        g_w = gate.reshape(-1)[a][:, None]
        s, se = DY @ w["o"][e].T, d * U32 * (np.abs(DY) @ np.abs(w["o"][e]).T)
        if act == "relu":
            h, he = Z, np.zeros_like(Z)
            slope, slope_e = [(Z > 0).astype(np.float64)], [np.zeros_like(Z)]
        else:
            g, u = np.split(Z, 2, axis=1)
            sig = sigmoid(g)
            h = g * sig * u
            # exp(-g) is off by (2 + |g|) roundings relatively, its reciprocal with 1 added by 2 more, and so on: 8 + 2 |g| cover all of them
            rel = (8 + 2 * np.abs(g)) * U32
            he = rel * np.abs(h)
            slope = [u * (sig + g * sig * (1 - sig)), g * sig]
            slope_e = [rel * np.abs(u) * (sig + 2 * np.abs(g) * sig), rel * np.abs(slope[1])]
        dgate[a] = (h * s).sum(1)
        dge[a] = (F * U32 * np.abs(h * s) + he * np.abs(s) + np.abs(h) * se).sum(1)
        wh = g_w * h
        whe = np.abs(g_w) * he + np.abs(wh) * (U16 + 2 * U32)
        n = len(a)
        out["o"][0][e] = wh.T @ DY
        out["o"][1][e] = whe.T @ np.abs(DY) + n * U32 * (np.abs(wh).T @ np.abs(DY))
        for name, sl_v, sl_e in zip("ab", slope, slope_e):
            dz = g_w * s * sl_v
            dze = np.abs(g_w) * (se * np.abs(sl_v) + np.abs(s) * sl_e) + np.abs(dz) * (U16 + 4 * U32)
            out[name][0][e] = X.T @ dz
            out[name][1][e] = np.abs(X).T @ dze + n * U32 * (np.abs(X).T @ np.abs(dz))
            dxp[sl] += dz @ w[name][e].T
            dxe[sl] += dze @ np.abs(w[name][e]).T + 2 * F * U32 * (np.abs(dz) @ np.abs(w[name][e]).T)
    return (dxp, dxe), (dgate, dge), out


def route_backward(logits, idx, gate, dgate, renorm):
    """dlogits [T,E]."""
    T, E = logits.shape
    dot = (gate * dgate).sum(1, keepdims=True)
    rows = np.arange(T)[:, None]
    if renorm:
        dl = np.zeros((T, E))
        dl[rows, idx] = gate * (dgate - dot)
        return dl
    p = np.exp(logits - logits.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    chosen = np.zeros((T, E))
    chosen[rows, idx] = dgate
    return p * (chosen - dot)
