"""The short convolution, the selective scan and the orthogonalised update in 64 bits (numpy), each with a bound on what
fp32 arithmetic may differ by, derived to first order from the formulas as in nets_ref.py: E is absolute, U the unit
roundoff of fp32."""
import numpy as np

from nets_ref import U, _ended, _sum_error, act, sigmoid


def conv_rows(x, K, state, done, done_prev):
    """[K, T, N, D]: what step t sees j rows back, and the new state."""
    T, N, D = x.shape
    z = np.concatenate([np.zeros((K - 1, N, D)) if state is None else state, x])
    end = _ended(T, N, done, done_prev)[..., 0]
    seen = np.zeros((K, T, N, D))
    left = np.zeros((K - 1, N, D))
    for n in range(N):
        last = -K                                        # the last step that an end came before
        for t in range(T):
            if end[t, n]:
                last = t
            for j in range(K):
                if t - j >= last:
                    seen[j, t, n] = z[K - 1 + t - j, n]
        for i in range(K - 1):
            if T - K + 1 + i >= last:
                left[i, n] = z[T + i, n]
    return seen, left


def conv(x, w, b, state, done, done_prev, name):
    """y, new_state and E of y."""
    K = w.shape[0]
    seen, left = conv_rows(x, K, state, done, done_prev)
    wj = w[::-1][:, None, None]                          # of the row j back
    p = (wj * seen).sum(0) + b
    Ep = (K + 2) * U * ((np.abs(wj * seen)).sum(0) + np.abs(b))
    y, _ = act(p, name)
    if name == "none":
        return y, left, Ep
    return y, left, 1.1 * Ep + U * (12 + np.abs(p)) * np.abs(y)


def conv_backward(x, w, b, dy, state, done, done_prev, dnew, name):
    """dx, dw, db, dstate and their E."""
    T, N, D = x.shape
    K = w.shape[0]
    seen, _ = conv_rows(x, K, state, done, done_prev)
    wj = w[::-1][:, None, None]
    p = (wj * seen).sum(0) + b
    Ep = (K + 2) * U * ((np.abs(wj * seen)).sum(0) + np.abs(b))
    slope = act(p, name)[1]
    dp = dy * slope
    Edp = np.zeros_like(dp) if name == "none" else np.abs(dy) * (0.5 * Ep + U * (14 + np.abs(p)) * (np.abs(slope) + 0.1))
    # which rows a step sees, from rows of ones (those of the state too)
    ones, left = conv_rows(np.ones_like(x), K, np.ones((K - 1, N, D)), done, done_prev)
    dz, Edz = np.zeros((T + K - 1, N, D)), np.zeros((T + K - 1, N, D))
    for j in range(K):
        s = slice(K - 1 - j, K - 1 - j + T)
        dz[s] += wj[j] * dp * ones[j]
        Edz[s] += np.abs(wj[j]) * (Edp + (K + 2) * U * np.abs(dp)) * ones[j]
    if dnew is not None:
        dz[T:] += dnew * left
        Edz[T:] += (K + 2) * U * np.abs(dnew * left)
    k = _sum_error(T * N)
    dw = (dp * seen).sum((1, 2))[::-1]
    Edw = (Edp * np.abs(seen)).sum((1, 2))[::-1] + k * np.abs(dp * seen).sum((1, 2))[::-1]
    return (dz[K - 1:], dw, dp.sum((0, 1)), dz[:K - 1], Edz[K - 1:], Edw,
            Edp.sum((0, 1)) + k * np.abs(dp).sum((0, 1)), Edz[:K - 1])


class Scan:
    """The forward pass, its states, and the bounds.  Arguments as select_scan's, arrays of 64 bits or None."""

    def __init__(self, x, dt, A, B, C, skip, bias, gate, h0, done, prev):
        T, N, D = x.shape
        S = A.shape[1]
        G = B.shape[2] // S
        self.sizes = T, N, D, S, G
        wide = lambda v: np.repeat(v.reshape(T, N, G, S), D // G, axis=2)     # noqa: E731  [T, N, D, S]
        self.B, self.C = wide(B), wide(C)
        self.x, self.A = x, A
        self.skip = np.zeros(D) if skip is None else skip
        v = dt + (0.0 if bias is None else bias)
        self.sig = sigmoid(v)
        self.e = np.logaddexp(0.0, v)
        # softplus: v rounded (U |v| times the slope), q = exp(-|v|) off by U (|v| + 4) of itself, the rest 8 units
        self.re = U * (12 + 2 * np.abs(v))                # relative
        self.gate = gate
        self.act, self.slope = (np.ones_like(x), np.zeros_like(x)) if gate is None else act(gate, "silu")
        self.end = _ended(T, N, done, prev)[..., None]
        self.h = np.zeros((T, N, D, S))
        self.c = np.zeros((T, N, D, S))                  # what step t continues from
        self.a = np.exp(self.e[..., None] * A)
        self.ra = U * 6 + np.abs(self.e[..., None] * A) * (self.re[..., None] + 3 * U)
        self.Eh = np.zeros((T, N, D, S))
        h = np.zeros((N, D, S)) if h0 is None else h0
        E = np.zeros((N, D, S))
        self.kept, self.Ekept = [], []
        for t in range(T):
            if t % 16 == 0:
                self.kept.append(h)
                self.Ekept.append(2 * E)
            h, E = np.where(self.end[t], 0.0, h), np.where(self.end[t], 0.0, E)
            self.c[t] = h
            into = (self.e[t] * x[t])[..., None] * self.B[t]
            E = self.a[t] * E + (self.ra[t] + 3 * U) * self.a[t] * np.abs(h) + (self.re[t][..., None] + 4 * U) * np.abs(into)
            h = self.a[t] * h + into
            self.h[t], self.Eh[t] = h, 2 * E             # twice: joins of pieces round products of decays instead
        self.hT, self.EhT = h, 2 * E
        terms = self.C * self.h
        self.p = terms.sum(-1) + self.skip * x
        self.Ep = (np.abs(self.C) * self.Eh).sum(-1) + (S + 4) * U * (np.abs(terms).sum(-1) + np.abs(self.skip * x))
        self.y = self.p * self.act
        self.ract = 0.0 if gate is None else U * (12 + np.abs(gate))
        self.Ey = np.abs(self.act) * (self.Ep + (self.ract + 2 * U) * np.abs(self.p))

    def backward(self, dy, dhT):
        """{name: (gradient, E)}."""
        T, N, D, S, G = self.sizes
        p = dy * self.act
        Ep = (self.ract + 2 * U) * np.abs(p)
        g = np.zeros((N, D, S)) if dhT is None else dhT
        Eg = np.zeros((N, D, S))
        f, Ef = np.zeros((T, N, D, S)), np.zeros((T, N, D, S))
        for t in reversed(range(T)):
            into = self.C[t] * p[t][..., None]
            f[t] = into + g
            Ef[t] = Eg + np.abs(self.C[t]) * Ep[t][..., None] + 2 * U * (np.abs(into) + np.abs(g))
            g = np.where(self.end[t], 0.0, self.a[t] * f[t])
            Eg = np.where(self.end[t], 0.0, self.a[t] * Ef[t] + (self.ra[t] + 3 * U) * np.abs(self.a[t] * f[t]))
        Ef = 2 * Ef
        out = {"dh0": (g, 2 * Eg)}
        e, x, re = self.e[..., None], self.x[..., None], self.re[..., None]
        past = self.a * self.c
        Epast = self.a * np.where(self.end, 0.0, np.concatenate([np.zeros((1, N, D, S)), self.Eh[:-1]])) + (self.ra + 2 * U) * np.abs(past)
        groups = lambda v: v.reshape(T, N, G, D // G, S).sum(3).reshape(T, N, G * S)      # noqa: E731
        kd = _sum_error(D // G) + 6 * U
        out["dC"] = (groups(p[..., None] * self.h),
                     groups(np.abs(p[..., None]) * self.Eh + Ep[..., None] * np.abs(self.h) + kd * np.abs(p[..., None] * self.h)))
        out["dB"] = (groups(e * x * f), groups(np.abs(e * x) * Ef + (re + kd) * np.abs(e * x * f)))
        Bf = (self.B * f).sum(-1)
        EBf = (np.abs(self.B) * Ef).sum(-1) + (S + 4) * U * np.abs(self.B * f).sum(-1)
        out["dx"] = (self.skip * p + self.e * Bf,
                     np.abs(self.skip) * (Ep + 3 * U * np.abs(p)) + self.e * (EBf + (self.re + 3 * U) * np.abs(Bf)))
        w = f * past
        Ew = Ef * np.abs(past) + np.abs(f) * Epast + 2 * U * np.abs(w)
        de = (w * self.A).sum(-1) + self.x * Bf
        Ede = ((Ew + 3 * U * np.abs(w)) * np.abs(self.A)).sum(-1) + (S + 4) * U * np.abs(w * self.A).sum(-1) + np.abs(self.x) * (EBf + 3 * U * np.abs(Bf))
        du = de * self.sig
        Edu = self.sig * (Ede + (self.re + 4 * U) * np.abs(de))
        out["ddt"] = (du, Edu)
        kt = _sum_error(T * N) + 6 * U
        out["ddt_bias"] = (du.sum((0, 1)), Edu.sum((0, 1)) + kt * np.abs(du).sum((0, 1)))
        out["dskip"] = ((p * self.x).sum((0, 1)), (Ep * np.abs(self.x)).sum((0, 1)) + kt * np.abs(p * self.x).sum((0, 1)))
        out["dA"] = ((w * e).sum((0, 1)), (Ew * e + (re + kt) * np.abs(w * e)).sum((0, 1)))
        if self.gate is not None:
            q = dy * self.slope
            Eq = np.abs(dy) * U * (14 + np.abs(self.gate)) * (np.abs(self.slope) + 0.1)
            out["dgate"] = (q * self.p, np.abs(q) * (self.Ep + 2 * U * np.abs(self.p)) + Eq * np.abs(self.p))
        return out


def orthogonalise(x, steps, coef, eps):
    """y [M, N] of one matrix, and a bound of the Frobenius norm of its error.

    A product of values in two pieces of 11 bits leaves 2^-22 of each term out and rounds each value by as much; its sum of K
    terms is added up 16 at a time for each of the three pieces' products, each addition off by at most 2^-23 (it may cut).  An
    error E of X goes through a step as p's divided differences on the singular values let it: at most max |p'|, |p / v|."""
    a, b, c = coef
    f = np.linalg.norm
    X = x / (f(x) + eps)
    E = (3 * 2.0 ** -22 + 8 * U) * f(X)
    fro_abs = lambda P, Q: f(np.abs(P) @ np.abs(Q))                # noqa: E731
    eta = lambda K: 4 * 2.0 ** -22 + 2.0 ** -23 * (3 * np.ceil(K / 64) * 4)     # noqa: E731
    for _ in range(steps):
        wide = X.shape[0] <= X.shape[1]
        Z = X if wide else X.T
        P = Z @ Z.T
        top = np.linalg.norm(X, 2) * 1.01
        EP = eta(Z.shape[1]) * fro_abs(Z, Z.T)
        Q = a * np.eye(len(P)) + b * P + c * P @ P
        EQ = (abs(b) + 2 * abs(c) * top ** 2) * EP + abs(c) * eta(len(P)) * fro_abs(P, P) + 4 * 2.0 ** -22 * f(Q)
        local = EQ * top + eta(len(P)) * fro_abs(Q, Z)
        v = np.linspace(0, top, 2001)
        grow = max(np.abs(a + 3 * b * v ** 2 + 5 * c * v ** 4).max(), np.abs(a + b * v ** 2 + c * v ** 4).max())
        E = grow * E + local
        X = Q @ X if wide else X @ Q
        E += 2.0 ** -22 * f(X)
    return X, E


# Sizes at which both pieces of X, of P and of Q weigh, and coefficients that give P P its part.
RANK_ONE = [(115, 110), (120, 125), (493, 874), (1044, 487), (493, 804), (518, 493), (991, 895), (613, 212), (630, 493), (493, 917)]
RANK_ONE_COEF = (0.2, 0.2, 0.6)


def _pieces(v):
    hi = np.float64(np.float16(v))
    return hi, np.float64(np.float16(v - hi))


def rank_one_update(M, N, steps, coef, lost=None):
    """One value of the update of a matrix of ones, whose result is v / sqrt(M N) everywhere, by the two fp16 pieces of each
    value and three products of them (scaled by 4096, 512 and 64), sums exact; lost: "P", "Q" or "X" and "hl" or "lh" for a
    product of pieces that is left out.  Every sum is of equal terms, so what a piece is to the result does not average out."""
    a, b, c = coef
    s, n = min(M, N), max(M, N)

    def product(u, v, which):
        (uh, ul), (vh, vl) = _pieces(u), _pieces(v)
        return uh * vh + (lost != which + "hl") * uh * vl + (lost != which + "lh") * ul * vh
    x = 4096 / np.sqrt(M * N)
    for _ in range(steps):
        p = n * product(x, x, "P") * 512 / 4096 ** 2
        q = b * sum(_pieces(p)) / 512 + c * s * product(p, p, "Q") / 512 ** 2
        x = ((s - 1) * product(64 * q, x, "X") + product(64 * (q + a), x, "X")) / 64
    return x / 4096


def rank_one_bound(M, N, steps, coef):
    """Relative bound of the same in fp32 and tensor products, for coefficients >= 0 that sum up to 1 (v stays 1, no sum
    cancels).  A value in two pieces is off by 2^-22 of itself and 2^-25 of its scaled unit; a product leaves 2^-22 of a term
    out, adds 16 terms in a tensor instruction and twelve of those to a sum over 64 of K, of which each may cut 2^-22 (those of
    the large pieces; the small ones' are 2^-11 of that), and rounds once for each 64 of K."""
    a, b, c = coef
    s, n = min(M, N), max(M, N)
    piece = lambda v: 2.0 ** -22 + 2.0 ** -25 / v                  # noqa: E731
    eta = lambda K: 13 * 2.0 ** -22 + np.ceil(K / 64) * U          # noqa: E731
    r = 80 * U                                                     # norm, a root of sums of up to 128 values in a row, and quotient
    for _ in range(steps):
        r += piece(4096 / np.sqrt(M * N))
        p = 2 * r + eta(n) + 4 * U + piece(512 / s)
        q = (b * p + c * (2 * p + eta(s))) / (b + c) + 4 * U + piece(64 * (b + c) / s)
        r += (b + c) * q + a * piece(64 * a) + eta(s) + 4 * U
    return r
