"""Measured cases of the state space memory and of what trains its weights: the short causal convolution, the selective
state space scan (each forward, as a single step, and backward) and the orthogonalised update of weight matrices.  ``run``
has each in plain torch operations, in 32 bits, and, where ``own`` is true, as calls of the framework's operators."""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
KEEP = 16                    # states are kept before every 16th step
COEF, EPS = (3.4445, -4.7750, 2.0315), 1e-7


# ------------------------------------------------------------------ cases
def listed():
    return [
        # One vehicle's control step through a 512-wide memory policy: latency.
        dict(name="conv_step_1", op="conv", T=1, N=1, D=512, K=4, act="silu", dtype="fp32", bias=True, done=True, state=True, pad=0),
        # Training pass over 128 steps of 4,096 envs, the value half of one projection.
        dict(name="conv_4096x128", op="conv", T=128, N=4096, D=256, K=4, act="silu", dtype="bf16", bias=True, done=True, state=True,
             pad=256),
        # Its gradient.
        dict(name="conv_back_4096x128", op="conv_back", T=128, N=4096, D=256, K=4, act="silu", dtype="bf16", bias=True, done=True,
             state=True, pad=256),
        # One vehicle's control step: latency.
        dict(name="scan_step_1", op="sscan", T=1, N=1, D=512, S=16, G=1, dtype="fp32", gate=True, done=True, h0=True, kept=False, fused=True),
        # One control step of the 65,536-env rollout, 256 wide: the states are what moves.
        dict(name="scan_step_65536", op="sscan", T=1, N=65536, D=256, S=16, G=1, dtype="bf16", gate=True, done=True, h0=True, kept=False,
             fused=True),
        # Training pass over 128 steps of 4,096 envs, states kept for the gradient.
        dict(name="scan_4096x128", op="sscan", T=128, N=4096, D=256, S=16, G=1, dtype="bf16", gate=True, done=True, h0=True, kept=True,
             fused=True),
        # One long log of a vehicle, odd length, odd widths, without a gate.
        dict(name="scan_long", op="sscan", T=65521, N=1, D=250, S=13, G=1, dtype="fp32", gate=False, done=False, h0=False, kept=False,
             fused=False),
        # Gradient of the training pass.
        dict(name="scan_back_4096x128", op="sscan_back", T=128, N=4096, D=256, S=16, G=1, dtype="bf16", gate=True, done=True, h0=True,
             kept=True, fused=True),
        # Gradient over a few long logs with episode ends, two groups of channels.
        dict(name="scan_back_long", op="sscan_back", T=8192, N=3, D=200, S=8, G=2, dtype="fp16", gate=True, done=True, h0=False, kept=True,
             fused=False),
        # Updates of a policy's and a critic's 256-wide layers: latency.
        dict(name="ortho_256", op="ortho", L=4, M=256, N=256, dtype="fp32", pad=0),
        # Projections of a stack of layers, odd sizes, rows of a wider array, momentum held in 16 bits.
        dict(name="ortho_stack", op="ortho", L=24, M=1000, N=515, dtype="bf16", pad=5),
        # One large matrix.
        dict(name="ortho_4096", op="ortho", L=1, M=4096, N=4096, dtype="fp32", pad=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["conv", "conv_back", "sscan", "sscan", "sscan_back", "sscan_back", "ortho", "ortho"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    if op in ("conv", "conv_back"):
        most = 60_000_000 if dtype != "fp32" else 30_000_000
        T, N, D = _log(rng, 1, 65536), _log(rng, 1, 65536), _log(rng, 1, 2048)
        if rng.random() < 0.6:          # widths are mostly round
            D = max(8, D // 8 * 8)
        N = max(1, min(N, most // D))
        T = max(1, min(T, most // (N * D)))
        return dict(op=op, T=T, N=N, D=D, K=rng.choice([1, 2, 3, 4, 4, 4, 5, 8]), act=rng.choice(["none", "silu", "silu"]), dtype=dtype,
                    bias=rng.random() < 0.7, done=rng.random() < 0.7, state=rng.random() < 0.7, pad=rng.choice([0, 0, 3, 8, D]))
    if op in ("sscan", "sscan_back"):
        most = 400_000_000              # states times steps
        G = rng.choice([1, 1, 1, 2, 4])
        S = rng.choice([1, 4, 8, 13, 16, 16, 16, 32, 64])
        D = G * _log(rng, 1, 1024 // G)
        if rng.random() < 0.6:
            D = max(8, D // G // 8 * 8) * G
        T, N = _log(rng, 1, 65536 if op == "sscan" else 8192), _log(rng, 1, 65536)
        N = max(1, min(N, most // (D * S)))
        T = max(1, min(T, most // (N * D * S)))
        return dict(op=op, T=T, N=N, D=D, S=S, G=G, dtype=dtype, gate=rng.random() < 0.7, done=rng.random() < 0.7, h0=rng.random() < 0.7,
                    kept=op == "sscan_back" or rng.random() < 0.5, fused=rng.random() < 0.5)
    while True:
        L, M, N = _log(rng, 1, 48), _log(rng, 1, 4096), _log(rng, 1, 4096)
        if rng.random() < 0.6:
            M, N = max(8, M // 8 * 8), max(8, N // 8 * 8)
        m, n = min(M, N), max(M, N)
        if 2 * L * m * m * n <= 1e11 and L * M * N <= 60_000_000:
            return dict(op=op, L=L, M=M, N=N, dtype=dtype, pad=rng.choice([0, 0, 0, 3, 8]))


# ------------------------------------------------------------------ inputs
def _normal(g, shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(shape, device="cuda", generator=g) * scale + shift).to(dtype)


def _padded(g, shape, pad, dtype, scale=1.0, shift=0.0):
    """Channels of a wider array: the last axis contiguous, rows `pad` elements further apart."""
    return _normal(g, (*shape[:-1], shape[-1] + pad), dtype, scale, shift)[..., :shape[-1]]


def _empty(shape, pad, dtype):
    return torch.empty((*shape[:-1], shape[-1] + pad), device="cuda", dtype=dtype)[..., :shape[-1]]


def _ends(st, case, g):
    T, N = case["T"], case["N"]
    st["done"] = st["done_prev"] = None
    if case["done"]:
        st["done"] = (torch.rand((T, N), device="cuda", generator=g) < 0.005).to(torch.uint8)
        st["done_prev"] = (torch.rand((N,), device="cuda", generator=g) < 0.1).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]
    st = dict(case=case)
    op = case["op"]
    f32 = torch.float32
    if op in ("conv", "conv_back"):
        T, N, D, K, pad = (case[k] for k in ("T", "N", "D", "K", "pad"))
        st["x"] = _padded(g, (T, N, D), pad, dt)
        st["w"] = _normal(g, (K, D), f32, K ** -0.5)
        st["bias"] = _normal(g, (D,), f32, 0.3) if case["bias"] else None
        st["state"] = _normal(g, (K - 1, N, D), dt) if case["state"] else None
        _ends(st, case, g)
        if op == "conv":
            st["y"] = torch.empty((T, N, D), device="cuda", dtype=dt)
            st["new_state"] = torch.empty((K - 1, N, D), device="cuda", dtype=dt)
        else:
            st["dy"] = _normal(g, (T, N, D), dt, 0.1)
            st["dnew_state"] = _normal(g, (K - 1, N, D), dt, 0.1)
            st["dx"] = _empty((T, N, D), pad, dt)
            st["dw"], st["dbias"] = torch.empty((K, D), device="cuda"), torch.empty((D,), device="cuda")
            st["dstate"] = torch.empty((K - 1, N, D), device="cuda", dtype=dt)
        return st
    if op in ("sscan", "sscan_back"):
        T, N, D, S, G = (case[k] for k in ("T", "N", "D", "S", "G"))
        if case["fused"]:               # x and gate: halves of one projection; B and C: of another
            z = _normal(g, (T, N, 2 * D), dt)
            st["x"], st["gate"] = z[..., :D], z[..., D:]
            z = _normal(g, (T, N, 2 * G * S), dt)
            st["B"], st["C"] = z[..., :G * S], z[..., G * S:]
        else:
            st["x"], st["gate"] = _normal(g, (T, N, D), dt), _normal(g, (T, N, D), dt)
            st["B"], st["C"] = _normal(g, (T, N, G * S), dt), _normal(g, (T, N, G * S), dt)
        if not case["gate"]:
            st["gate"] = None
        st["dt"] = _normal(g, (T, N, D), dt, 0.5)
        # step sizes of 0.001 to 0.1 about their bias, rates of 1 to S: memories of some steps to thousands
        step = torch.exp(torch.rand((D,), device="cuda", generator=g) * math.log(100) + math.log(1e-3))
        st["dt_bias"] = step + torch.log(-torch.expm1(-step))
        st["A"] = -torch.exp(torch.log(torch.arange(1, S + 1, device="cuda", dtype=f32)) + _normal(g, (D, S), f32, 0.1))
        st["skip"] = _normal(g, (D,), f32, 0.2, 1.0)
        _ends(st, case, g)
        st["h0"] = _normal(g, (N, D, S), f32, 0.3) if case["h0"] else None
        kept = ((T + KEEP - 1) // KEEP, N, D, S)
        if op == "sscan":
            st["y"] = torch.empty((T, N, D), device="cuda", dtype=dt)
            st["hT"] = torch.empty((N, D, S), device="cuda")
            st["kept"] = torch.empty(kept, device="cuda") if case["kept"] else None
        else:
            st["kept"] = torch.empty(kept, device="cuda")       # as the forward pass leaves them
            _plain_sscan(st, want_y=False)
            st["dy"] = _normal(g, (T, N, D), dt, 0.1)
            st["dhT"] = _normal(g, (N, D, S), f32, 0.1)
            for k in ("x", "dt", "gate", "B", "C"):
                st["d" + k] = None if st[k] is None else torch.empty(st[k].shape, device="cuda", dtype=dt)
            for k in ("A", "skip", "dt_bias"):
                st["d" + k] = torch.empty_like(st[k])
            st["dh0"] = torch.empty((N, D, S), device="cuda")
        return st
    L, M, N = case["L"], case["M"], case["N"]
    # an update: a few strong directions over noise
    r = max(1, min(M, N) // 8)
    x = _normal(g, (L, M, r), f32, r ** -0.5) @ _normal(g, (L, r, N), f32) + _normal(g, (L, M, N), f32, 0.5)
    st["x"] = _empty((L, M, N), case["pad"], dt)
    st["x"].copy_(x * 1e-3)
    st["y"] = torch.empty((L, M, N), device="cuda", dtype=dt)
    return st


# ------------------------------------------------------------------ plain forms
def _ended(st, T, N):
    """[T, N]: whether an episode ended before step t."""
    if st["done"] is None:
        return torch.zeros((T, N), dtype=torch.bool, device="cuda")
    return torch.cat([st["done_prev"][None], st["done"][:-1]]).bool()


def _silu(u):
    """silu(u) and its derivative."""
    s = torch.sigmoid(u)
    return u * s, s * (1 + u * torch.sigmoid(-u))


def _reach(end, j):
    """[T, N, 1]: whether step t still sees the row j steps before it."""
    T = end.shape[0]
    ok = torch.ones_like(end)
    for i in range(min(j, T)):          # an end before step t, t - 1, ... cuts it off
        ok[i:] &= ~end[:T - i]
    return ok[..., None]


def _plain_conv_parts(st):
    """Inputs with the state in front, what step t sees of them j rows back, and the sums."""
    x = st["x"].float()
    T, N, D = x.shape
    K = st["w"].shape[0]
    before = torch.zeros((K - 1, N, D), device="cuda") if st["state"] is None else st["state"].float()
    z = torch.cat([before, x])
    reach = [_reach(_ended(st, T, N), j) for j in range(K)]
    seen = lambda j: torch.where(reach[j], z[K - 1 - j:K - 1 - j + T], 0.0)    # noqa: E731
    p = torch.zeros((T, N, D), device="cuda")
    for j in range(K - 1, -1, -1):
        p += st["w"][K - 1 - j] * seen(j)
    if st["bias"] is not None:
        p += st["bias"]
    return z, reach, seen, p


def _left(st, K, T, N):
    """[K - 1, N, 1]: which of the last K - 1 rows (state and inputs) no episode end before the last step cuts off."""
    end = _ended(st, T, N)
    rows = torch.arange(T - K + 1, T, device="cuda")[:, None]          # their steps; below 0 the state's
    last = torch.where(end, torch.arange(T, device="cuda")[:, None], -K).amax(dim=0)[None]
    return (rows >= last)[..., None]


def _plain_conv(st):
    z, _, _, p = _plain_conv_parts(st)
    T, N, D = p.shape
    K = st["w"].shape[0]
    y = _silu(p)[0] if st["case"]["act"] == "silu" else p
    t = st["x"].dtype
    return y.to(t), torch.where(_left(st, K, T, N), z[T:], 0.0).to(t)


def _plain_conv_back(st):
    z, reach, seen, p = _plain_conv_parts(st)
    T, N, D = p.shape
    K = st["w"].shape[0]
    dp = st["dy"].float()
    if st["case"]["act"] == "silu":
        dp = dp * _silu(p)[1]
    dz = torch.zeros((T + K - 1, N, D), device="cuda")
    dw = torch.empty((K, D), device="cuda")
    for j in range(K):
        dz[K - 1 - j:K - 1 - j + T] += torch.where(reach[j], st["w"][K - 1 - j] * dp, 0.0)
        dw[K - 1 - j] = (dp * seen(j)).sum(dim=(0, 1))
    dz[T:] += torch.where(_left(st, K, T, N), st["dnew_state"].float(), 0.0)
    t = st["x"].dtype
    return dz[K - 1:].to(t), dw, dp.sum(dim=(0, 1)), dz[:K - 1].to(t)


def _softplus(u):
    return torch.clamp_min(u, 0.0) + torch.log1p(torch.exp(-torch.abs(u)))


def _doubling(A, X):
    """h_t = A_t h_{t-1} + X_t along the first axis (h before it 0): after a round each element holds its last 2, 4, 8, ...
    steps.  Exact zeros of A cut the past off."""
    s = 1
    while s < X.shape[0]:
        X = torch.cat([X[:s], torch.where(A[s:] == 0, X[s:], A[s:] * X[:-s] + X[s:])])
        A = torch.cat([A[:s], A[s:] * A[:-s]])
        s *= 2
    return X


class _Parts:
    """The scan's inputs in 32 bits, channels as [G, D / G]."""

    def __init__(self, st):
        case = st["case"]
        T, N, D, S, G = (case[k] for k in ("T", "N", "D", "S", "G"))
        self.sizes = T, N, D, S, G
        self.x = st["x"].float().reshape(T, N, G, D // G)
        self.u = (st["dt"].float() + st["dt_bias"]).view(T, N, G, D // G)
        self.step = _softplus(self.u)
        self.B, self.C = (st[k].float().reshape(T, N, G, S) for k in ("B", "C"))
        self.A = st["A"].view(G, D // G, S)
        self.skip = st["skip"].view(G, D // G)
        self.gate = None if st["gate"] is None else st["gate"].float().reshape(T, N, G, D // G)
        self.end = _ended(st, T, N)[..., None, None, None]
        self.h0 = torch.zeros((N, G, D // G, S), device="cuda") if st["h0"] is None else st["h0"].view(N, G, D // G, S)

    def decay(self, t):
        return torch.exp(self.step[t][..., None] * self.A)

    def into(self, t):
        return (self.step[t] * self.x[t])[..., None] * self.B[t][..., None, :]


def _plain_states(q):
    """[T, N, G, D / G, S] states, by doubling: for long sequences."""
    every = slice(None)
    a, X = torch.where(q.end, 0.0, q.decay(every)), q.into(every)
    X[0] += torch.where(q.end[0], 0.0, a[0] * q.h0)
    return _doubling(a, X)


def _plain_sscan(st, want_y=True):
    q = _Parts(st)
    T, N, D, S, G = q.sizes
    p = torch.empty_like(q.x)
    kept = st["kept"]
    if T > 1024:
        h = _plain_states(q)
        p = (h * q.C[..., None, :]).sum(-1)
        last = h[-1].clone()
        if kept is not None:
            kept[0] = q.h0.view(N, D, S)
            kept[1:] = h[KEEP - 1:T - 1:KEEP].reshape(-1, N, D, S)
    else:
        last = q.h0
        for t in range(T):
            if kept is not None and t % KEEP == 0:
                kept[t // KEEP] = last.reshape(N, D, S)
            last = q.decay(t) * torch.where(q.end[t], 0.0, last) + q.into(t)
            if want_y:
                p[t] = (last * q.C[t][..., None, :]).sum(-1)
    if not want_y:
        return None
    p = p + q.skip * q.x
    if q.gate is not None:
        p = p * _silu(q.gate)[0]
    return p.reshape(T, N, D).to(st["x"].dtype), last.reshape(N, D, S), *(() if kept is None else (kept,))


def _plain_sscan_back(st):
    q = _Parts(st)
    T, N, D, S, G = q.sizes
    dy = st["dy"].float().view(q.x.shape)
    dp = dy
    if q.gate is not None:
        act, slope = _silu(q.gate)
        dp = dy * act
    g = st["dhT"].view(q.h0.shape)
    if T > 1024:
        h = _plain_states(q)
        keep = torch.where(q.end, 0.0, q.decay(slice(None)))
        X = dp[..., None] * q.C[..., None, :]
        X[-1] += g
        grad = _doubling(torch.cat([keep[1:], torch.zeros_like(keep[:1])]).flip(0), X.flip(0)).flip(0)
        passed = keep * torch.cat([torch.where(q.end[:1], 0.0, q.h0[None]), h[:-1]])        # a c
        y = (h * q.C[..., None, :]).sum(-1)
        dC = (h * dp[..., None]).sum(3)
        dB = (grad * (q.step * q.x)[..., None]).sum(3)
        Bg = (grad * q.B[..., None, :]).sum(-1)
        dstep = (grad * passed * q.A).sum(-1)
        dA = (grad * passed * q.step[..., None]).sum(dim=(0, 1))
        g = keep[0] * grad[0]
    else:
        h = torch.empty((T, *q.h0.shape), device="cuda")
        last = q.h0
        for t in range(T):
            last = torch.add(q.decay(t) * torch.where(q.end[t], 0.0, last), q.into(t), out=h[t])
        y, Bg, dstep = (torch.empty_like(q.x) for _ in range(3))
        dB, dC = torch.empty_like(q.B), torch.empty_like(q.C)
        dA = torch.zeros_like(q.A)
        for t in reversed(range(T)):
            y[t] = (h[t] * q.C[t][..., None, :]).sum(-1)
            grad = g + dp[t][..., None] * q.C[t][..., None, :]
            decay = q.decay(t)
            passed = grad * torch.where(q.end[t], 0.0, decay * (h[t - 1] if t else q.h0))
            dC[t] = (h[t] * dp[t][..., None]).sum(2)
            dB[t] = (grad * (q.step[t] * q.x[t])[..., None]).sum(2)
            Bg[t] = (grad * q.B[t][..., None, :]).sum(-1)
            dstep[t] = (passed * q.A).sum(-1)
            dA += (passed * q.step[t][..., None]).sum(0)
            g = torch.where(q.end[t], 0.0, decay * grad)
    dx = q.skip * dp + q.step * Bg
    du = (dstep + q.x * Bg) * torch.sigmoid(q.u)
    t = st["x"].dtype
    flat = lambda v: v.reshape(T, N, -1).to(t)                                   # noqa: E731
    dgate = None if q.gate is None else flat(dy * (y + q.skip * q.x) * slope)
    return (flat(dx), flat(du), dA.reshape(D, S), flat(dB), flat(dC), (dp * q.x).sum(dim=(0, 1)).view(D),
            du.sum(dim=(0, 1)).view(D), dgate, g.reshape(N, D, S))


def _plain_ortho(st):
    x = st["x"].float()
    turned = x.shape[1] > x.shape[2]
    if turned:
        x = x.transpose(1, 2)
    x = x / (torch.sqrt((x * x).sum(dim=(1, 2), keepdim=True)) + EPS)
    a, b, c = COEF
    for _ in range(5):
        P = x @ x.transpose(1, 2)
        x = a * x + (b * P + c * (P @ P)) @ x
    return (x.transpose(1, 2) if turned else x).to(st["x"].dtype).contiguous()


# ------------------------------------------------------------------ one pass
def run(st):
    op = st["case"]["op"]
    if not own:
        return {"conv": _plain_conv, "conv_back": _plain_conv_back, "sscan": _plain_sscan, "sscan_back": _plain_sscan_back,
                "ortho": _plain_ortho}[op](st)
    from paper_2512_13359_gb300 import nets
    if op == "conv":
        return nets.causal_conv(st["x"], st["w"], st["bias"], st["state"], done=st["done"], done_prev=st["done_prev"],
                                act=st["case"]["act"], y=st["y"], new_state=st["new_state"])
    if op == "conv_back":
        return nets.causal_conv_backward(st["x"], st["w"], st["bias"], st["dy"], st["state"], done=st["done"], done_prev=st["done_prev"],
                                         act=st["case"]["act"], dnew_state=st["dnew_state"], dx=st["dx"], dw=st["dw"],
                                         dbias=st["dbias"], dstate=st["dstate"])
    if op == "sscan":
        out = nets.select_scan(st["x"], st["dt"], st["A"], st["B"], st["C"], skip=st["skip"], dt_bias=st["dt_bias"], gate=st["gate"],
                               h0=st["h0"], done=st["done"], done_prev=st["done_prev"], y=st["y"], hT=st["hT"], kept=st["kept"])
        return out if st["kept"] is not None else out[:2]
    if op == "sscan_back":
        return nets.select_scan_backward(st["x"], st["dt"], st["A"], st["B"], st["C"], st["kept"], st["dy"], skip=st["skip"],
                                         dt_bias=st["dt_bias"], gate=st["gate"], done=st["done"], done_prev=st["done_prev"],
                                         dhT=st["dhT"], dx=st["dx"], ddt=st["ddt"], dA=st["dA"], dB=st["dB"], dC=st["dC"],
                                         dskip=st["dskip"], ddt_bias=st["ddt_bias"], dgate=st["dgate"], dh0=st["dh0"])
    return nets.orthogonalise(st["x"], 5, coef=COEF, eps=EPS, y=st["y"])


def work(case):
    """Bytes: each input once, each output once.  Operations: of the formulas, an exponential or a division as one; a
    symmetric product as its half."""
    op, z = case["op"], SIZE[case["dtype"]]
    if op in ("conv", "conv_back"):
        T, N, D, K = (case[k] for k in ("T", "N", "D", "K"))
        n, m = T * N * D, (K - 1) * N * D
        states = m * z * ((1 if op == "conv" else 2) + case["state"])
        ends = (T * N + N) if case["done"] else 0
        act = case["act"] == "silu"
        return {"bytes": n * z * (2 if op == "conv" else 3) + states + ends + 4 * (K + 1) * D * (1 if op == "conv" else 2),
                "flops": n * (2 * K + 4 * act if op == "conv" else 4 * K + act * (2 * K + 8))}
    if op in ("sscan", "sscan_back"):
        T, N, D, S, G = (case[k] for k in ("T", "N", "D", "S", "G"))
        n, m, rows = T * N * D, N * D * S, T * N * G * S
        ends = (T * N + N) if case["done"] else 0
        kept = 4 * m * ((T + KEEP - 1) // KEEP) if case["kept"] else 0
        if op == "sscan":
            return {"bytes": n * z * (3 + case["gate"]) + 2 * rows * z + 4 * m * (1 + case["h0"]) + kept + ends + 4 * D * (S + 2),
                    "flops": n * (7 * S + 8)}
        return {"bytes": n * z * (5 + 2 * case["gate"]) + 4 * rows * z + 8 * m + kept + ends + 8 * D * (S + 2),
                "flops": n * (20 * S + 20)}
    L, m, n = case["L"], min(case["M"], case["N"]), max(case["M"], case["N"])
    return {"bytes": 2 * L * m * n * z, "flops": L * 5 * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)}


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    with torch.enable_grad():
        return {"conv": _exact_conv, "conv_back": _exact_conv_back, "sscan": _exact_sscan, "sscan_back": _exact_sscan_back,
                "ortho": _exact_ortho}[case["op"]](st)


def _flag(st, t, part):
    """[n, 1] of the envs of `part`: an episode ended before step t."""
    return (st["done_prev"][part] if t == 0 else st["done"][t - 1, part]).bool()[:, None]


def _conv_steps(st, x, w, bias, window, part):
    """Outputs of the steps, and the window after the last: the last K - 1 rows, 0 where an episode has ended since."""
    ys = []
    for t in range(x.shape[0]):
        if st["done"] is not None:
            e = _flag(st, t, part)
            window = [r.masked_fill(e, 0.0) for r in window]
        rows = [*window, x[t]]
        p = sum(r * k for r, k in zip(rows, w)) + bias
        ys.append(p / (1 + torch.exp(-p)) if st["case"]["act"] == "silu" else p)
        window = rows[1:]
    return torch.stack(ys), window


def _slices(N, each, limit):
    """Slices of the envs so that `each` values an env stay below `limit` in one."""
    k = max(1, min(N, limit // max(1, each)))
    return [slice(i, min(i + k, N)) for i in range(0, N, k)]


def _exact_conv(st):
    T, N, D = st["x"].shape
    K = st["w"].shape[0]
    w = list(st["w"].double())
    bias = 0.0 if st["bias"] is None else st["bias"].double()
    ys, ends = [], []
    for s in _slices(N, T * D, 200_000_000):
        k = s.stop - s.start
        window = list(torch.zeros((K - 1, k, D), dtype=torch.float64, device="cuda") if st["state"] is None else st["state"][:, s].double())
        y, window = _conv_steps(st, st["x"][:, s].double(), w, bias, window, s)
        ys.append(y)
        ends.append(torch.stack(window) if window else torch.zeros((0, k, D), dtype=torch.float64, device="cuda"))
    return torch.cat(ys, dim=1), torch.cat(ends, dim=1)


def _exact_conv_back(st):
    T, N, D = st["x"].shape
    K = st["w"].shape[0]
    w = st["w"].double().requires_grad_()
    b = (torch.zeros(D, device="cuda") if st["bias"] is None else st["bias"]).double().requires_grad_()
    dx, ds, dw, db = [], [], 0.0, 0.0
    for s in _slices(N, T * D, 30_000_000):
        x = st["x"][:, s].double().requires_grad_()
        st0 = (torch.zeros((K - 1, s.stop - s.start, D), device="cuda") if st["state"] is None else st["state"][:, s]).double().requires_grad_()
        y, window = _conv_steps(st, x, w.unbind(), b, list(st0.unbind()), s)
        loss = (y * st["dy"][:, s].double()).sum()
        if K > 1:
            loss = loss + (torch.stack(window) * st["dnew_state"][:, s].double()).sum()
        g = torch.autograd.grad(loss, (x, w, b, st0), allow_unused=True)
        dx.append(g[0])
        dw, db = dw + g[1], db + g[2]
        ds.append(torch.zeros_like(st0) if g[3] is None else g[3])
    return torch.cat(dx, dim=1), dw, db, torch.cat(ds, dim=1)


def _scan_step(st, t, part, h, x, u, A, B, C, skip, gate):
    """One step of the definition over envs `part`, everything in 64 bits: x, u, gate [n, D], B, C [n, G, S]."""
    n, D = x.shape
    G = B.shape[1]
    if st["done"] is not None:
        h = h.masked_fill(_flag(st, t, part)[..., None], 0.0)
    step = torch.where(u > 30, u, torch.log1p(torch.exp(torch.clamp_max(u, 30))))
    wide = lambda v: v[:, :, None].expand(n, G, D // G, -1).reshape(n, D, -1)    # noqa: E731
    h = torch.addcmul((step * x)[..., None] * wide(B), torch.exp(step[..., None] * A), h)
    y = torch.einsum("nds,nds->nd", h, wide(C)) + skip * x
    return h, y if gate is None else y * gate / (1 + torch.exp(-gate))


def _exact_sscan(st):
    case = st["case"]
    T, N, D, S, G = (case[k] for k in ("T", "N", "D", "S", "G"))
    A, bias, skip = (st[k].double() for k in ("A", "dt_bias", "skip"))
    h = torch.zeros((N, D, S), dtype=torch.float64, device="cuda") if st["h0"] is None else st["h0"].double()
    y = torch.empty((T, N, D), dtype=torch.float64, device="cuda")
    every, kept = slice(0, N), []
    for t in range(T):
        if t % KEEP == 0 and case["kept"]:
            kept.append(h)
        h, y[t] = _scan_step(st, t, every, h, st["x"][t].double(), st["dt"][t].double() + bias, A, st["B"][t].double().view(N, G, S),
                             st["C"][t].double().view(N, G, S), skip, None if st["gate"] is None else st["gate"][t].double())
    return (y, h, torch.stack(kept)) if case["kept"] else (y, h)


def _exact_sscan_back(st):
    """By differentiation of the steps, a few envs at a time and, of those, from one kept state to the next."""
    case = st["case"]
    T, N, D, S, G = (case[k] for k in ("T", "N", "D", "S", "G"))
    A, bias, skip = (st[k].double().requires_grad_() for k in ("A", "dt_bias", "skip"))
    names = ("x", "dt", "B", "C", "gate")
    per = {k: None if st[k] is None else torch.empty(st[k].shape, dtype=torch.float64, device="cuda") for k in names}
    sums = [torch.zeros_like(v) for v in (A, bias, skip)]
    dh0 = torch.empty((N, D, S), dtype=torch.float64, device="cuda")
    for s in _slices(N, KEEP * D * S, 100_000_000):
        n = s.stop - s.start
        h = torch.zeros((n, D, S), dtype=torch.float64, device="cuda") if st["h0"] is None else st["h0"][s].double()

        def steps(t0, h, v):
            ys = []
            for i in range(min(KEEP, T - t0)):
                gate = None if v["gate"] is None else v["gate"][i]
                h, y = _scan_step(st, t0 + i, s, h, v["x"][i], v["dt"][i] + bias, A, v["B"][i].view(n, G, S), v["C"][i].view(n, G, S),
                                  skip, gate)
                ys.append(y)
            return h, torch.stack(ys)

        def inputs(t0):
            return {k: None if st[k] is None else st[k][t0:t0 + KEEP, s].double().requires_grad_() for k in names}
        starts = []
        with torch.no_grad():
            for t0 in range(0, T, KEEP):
                starts.append(h)
                h, _ = steps(t0, h, inputs(t0))
        g = st["dhT"][s].double()
        for t0 in reversed(range(0, T, KEEP)):
            v = inputs(t0)
            h = starts.pop().detach().requires_grad_()
            end, y = steps(t0, h, v)
            loss = (y * st["dy"][t0:t0 + KEEP, s].double()).sum() + (end * g).sum()
            live = [k for k in names if v[k] is not None]
            grads = torch.autograd.grad(loss, [A, bias, skip, h, *(v[k] for k in live)])
            for total, part in zip(sums, grads):
                total += part
            g = grads[3]
            for k, q in zip(live, grads[4:]):
                per[k][t0:t0 + KEEP, s] = q
        dh0[s] = g
    return per["x"], per["dt"], sums[0], per["B"], per["C"], sums[2], sums[1], per["gate"], dh0


def _exact_ortho(st):
    a, b, c = COEF
    x = st["x"].double()
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + EPS)
    wide = x.shape[1] <= x.shape[2]
    for _ in range(5):          # on the shorter side; the other order of the products is the same polynomial
        q = torch.matmul(x, x.mT) if wide else torch.matmul(x.mT, x)
        r = torch.matmul(q, q).mul_(c).add_(q, alpha=b)
        r.diagonal(dim1=1, dim2=2).add_(a)
        x = torch.matmul(r, x) if wide else torch.matmul(x, r)
    return x
