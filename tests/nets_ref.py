"""The network operators in 64 bits (numpy), each with a bound on what fp32 arithmetic may differ by, derived to first
order from the formulas: E below is absolute, `u` the unit roundoff of fp32.  A result stored in 16 bits is rounded once
more (`stored`)."""
import numpy as np

U = 2.0 ** -24
ROUND = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # half a unit in the last place, or more
TINY = {"fp32": 2.0 ** -126, "bf16": 2.0 ** -126, "fp16": 2.0 ** -24}   # smallest step near 0 (fp16: subnormal)


def stored(ref, E, dtype):
    """Bound of a stored result: its error and one rounding of a value that much off."""
    return E + ROUND[dtype] * (np.abs(ref) + E) + TINY[dtype]


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def _gate(f):
    """a, 1 - a and the relative error of either in fp32: an exponential of an argument rounded to u |f| (and 2 ulp of
    its own, 4 u), a sum, a reciprocal (2 ulp) and a product: u (|f| + 12)."""
    a, b = sigmoid(f), sigmoid(-f)
    return a, b, U * (np.minimum(np.abs(f), 100.0) + 12.0)


def _ended(T, N, done, done_prev):
    e = np.zeros((T, N, 1), bool)
    if done is not None:
        e[1:, :, 0] = done[:-1] != 0
    if done_prev is not None and T:
        e[0, :, 0] = done_prev != 0
    return e


def gate_scan(f, v, h0, done, done_prev):
    """y, hT and E of y and of hT.  Each step adds relative errors of its two products and of its sum (3 u) to what the
    step before left, which its gate scales.  A scan that joins pieces of the sequence rounds each product of gates
    instead, the same errors to first order; twice the bound leaves room for the joins' own."""
    T, N, D = f.shape
    h = np.zeros((N, D)) if h0 is None else h0.astype(np.float64)
    E = np.zeros((N, D))
    y, Ey = np.zeros((T, N, D)), np.zeros((T, N, D))
    end = _ended(T, N, done, done_prev)
    for t in range(T):
        a, b, r = _gate(f[t])
        h, E = np.where(end[t], 0.0, h), np.where(end[t], 0.0, E)
        E = a * E + (r + 3 * U) * (a * np.abs(h) + b * np.abs(v[t]))
        h = a * h + b * v[t]
        y[t], Ey[t] = h, 2 * E
    return y, h, Ey, 2 * E


def gate_scan_backward(f, v, y, dy, h0, done, done_prev, dhT):
    """df, dv, dh0 and their E."""
    T, N, D = f.shape
    g = np.zeros((N, D)) if dhT is None else dhT.astype(np.float64)
    E = np.zeros((N, D))
    z = np.zeros((N, D)) if h0 is None else h0.astype(np.float64)
    end = _ended(T, N, done, done_prev)
    df, dv, Edf, Edv = (np.zeros((T, N, D)) for _ in range(4))
    for t in reversed(range(T)):
        a, b, r = _gate(f[t])
        c = np.where(end[t], 0.0, y[t - 1] if t else z)
        d = dy[t] + g
        E = E + 2 * U * (np.abs(dy[t]) + np.abs(g))
        dv[t], Edv[t] = b * d, b * (2 * E + (r + 3 * U) * np.abs(d))
        df[t] = a * b * (c - v[t]) * d
        Edf[t] = a * b * (np.abs(c - v[t]) * 2 * E + (2 * r + 6 * U) * (np.abs(c) + np.abs(v[t])) * np.abs(d))
        g = np.where(end[t], 0.0, a * d)
        E = np.where(end[t], 0.0, a * E + (r + 3 * U) * np.abs(a * d))
    return df, dv, g, Edf, Edv, 2 * E


ACTS = ("none", "relu", "silu", "tanh")


def act(u, name):
    """act(u), act'(u)."""
    if name == "relu":
        return np.maximum(u, 0.0), (u > 0).astype(np.float64)
    if name == "silu":
        s = sigmoid(u)
        return u * s, s * (1 + u * (1 - s))
    if name == "tanh":
        return np.tanh(u), 1 - np.tanh(u) ** 2
    return u, np.ones_like(u)


def _sum_error(n):
    """Relative to the sum of magnitudes, of n terms added in fp32 by at least 128 running sums that are then joined:
    roundings are as often up as down, so a chain of k additions drifts by some sqrt(k) u; 4 of those and the tree."""
    return U * (24 + 4 * np.sqrt(n / 128))


def _split(x, G):
    B, S, C = x.shape
    return x.reshape(B, S, G, C // G)


def group_norm(x, G, gamma, beta, eps, name):
    """y, mean, rstd and their E."""
    B, S, C = x.shape
    xg = _split(x, G)
    n = S * (C // G)
    k = _sum_error(n)
    mean = xg.mean(axis=(1, 3))
    dev = xg - mean[:, None, :, None]
    var = (dev ** 2).mean(axis=(1, 3))
    rstd = 1 / np.sqrt(var + eps)
    Em = k * np.abs(xg).mean(axis=(1, 3))
    # the deviations are off by Em each, which their square's mean feels to second order, and by a rounding; a variance
    # joined from pieces squares the distances of the pieces' means, with those means' errors: 2 Em sqrt(var)
    Ev = (k + 8 * U) * var + Em ** 2 + 2 * Em * np.sqrt(var)
    Er = rstd * (0.5 * Ev / (var + eps) + 6 * U)
    xh = (dev * rstd[:, None, :, None]).reshape(B, S, C)
    Exh = ((Em[:, None, :, None] + 2 * U * np.abs(dev)) * rstd[:, None, :, None]
           + np.abs(dev) * Er[:, None, :, None]).reshape(B, S, C)
    u = gamma * xh + beta
    Eu = np.abs(gamma) * Exh + 3 * U * (np.abs(gamma * xh) + np.abs(beta))
    y, _ = act(u, name)
    # slopes are at most 1.1; the function's own error: 8 u, and silu's exponential by its argument
    return y, mean, rstd, 1.1 * Eu + U * (8 + np.abs(u)) * np.abs(y) + 2 * U * (name == "tanh"), Em, Er


def group_norm_backward(x, G, gamma, beta, mean, rstd, dy, name):
    """dx, dgamma, dbeta and their E, from the given mean and rstd."""
    B, S, C = x.shape
    n = S * (C // G)
    m, r = mean[:, None, :, None], rstd[:, None, :, None]
    xh = ((_split(x, G) - m) * r).reshape(B, S, C)
    Exh = (2 * U * (np.abs(_split(x, G)) + np.abs(m)) * r).reshape(B, S, C) + U * np.abs(xh)
    u = gamma * xh + beta
    Eu = np.abs(gamma) * Exh + 3 * U * (np.abs(gamma * xh) + np.abs(beta))
    slope = act(u, name)[1]
    dz = dy * slope
    curve = 0.0 if name in ("none", "relu") else 1.0           # |act''| <= 1 for silu and tanh
    Edz = np.abs(dy) * (curve * Eu + U * (10 + np.abs(u)) * (curve + np.abs(slope)))
    w, Ew = gamma * dz, np.abs(gamma) * (Edz + U * np.abs(dz))
    wg, xg, Ewg, Exg = (_split(q, G) for q in (w, xh, Ew, Exh))
    k = _sum_error(n)
    avg = lambda q: q.mean(axis=(1, 3), keepdims=True)         # noqa: E731
    m1, m2 = avg(wg), avg(wg * xg)
    E1 = avg(Ewg) + k * avg(np.abs(wg))
    E2 = avg(Ewg * np.abs(xg) + np.abs(wg) * Exg) + k * avg(np.abs(wg * xg))
    dx = r * (wg - m1 - xg * m2)
    Edx = r * (Ewg + E1 + np.abs(xg) * E2 + np.abs(m2) * Exg
               + 4 * U * (np.abs(wg) + np.abs(m1) + np.abs(xg * m2)))
    kb = _sum_error(B * S)
    dbeta, dgamma = dz.sum(axis=(0, 1)), (dz * xh).sum(axis=(0, 1))
    Edb = Edz.sum(axis=(0, 1)) + kb * np.abs(dz).sum(axis=(0, 1))
    Edg = (Edz * np.abs(xh) + np.abs(dz) * Exh).sum(axis=(0, 1)) + kb * np.abs(dz * xh).sum(axis=(0, 1))
    return dx.reshape(B, S, C), dgamma, dbeta, Edx.reshape(B, S, C), Edg, Edb


def philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 words, [n, 4], of counters given as arrays or numbers."""
    m = np.uint64(0xFFFFFFFF)
    c = [np.atleast_1d(np.asarray(q, dtype=np.uint64)) for q in (c0, c1, c2, c3)]
    c = list(np.broadcast_arrays(*c))
    for r in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        ka = np.uint64((k0 + r * 0x9E3779B9) & 0xFFFFFFFF)
        kb = np.uint64((k1 + r * 0xBB67AE85) & 0xFFFFFFFF)
        s = np.uint64(32)
        c = [(b >> s) ^ c[1] ^ ka, b & m, (a >> s) ^ c[3] ^ kb, a & m]
    return np.stack(c, axis=-1).astype(np.uint32)


def dropout_keep(n, p, seed, draw):
    """[n] of 0 or 1 / (1 - p)."""
    thr = int(np.floor(p * 65536 + 0.5))
    q = np.arange((n + 7) // 8, dtype=np.uint64)
    w = philox(q & np.uint64(0xFFFFFFFF), q >> np.uint64(32), draw & 0xFFFFFFFF, draw >> 32, seed & 0xFFFFFFFF,
               seed >> 32)
    bits = np.stack([w & 0xFFFF, w >> 16], axis=-1).reshape(-1)[:n]
    return np.where(bits < thr, 0.0, 65536.0 / max(65536 - thr, 1))
