"""Measured cases of the network operators: the gated linear recurrence (forward, one step, backward), group norm with
an activation (forward and backward) and counter-based dropout.  ``run`` has each in plain torch operations, in 32 bits,
and, where ``own`` is true, as calls of the framework's operators."""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


# ------------------------------------------------------------------ cases
def listed():
    return [
        # One vehicle's control step through a 256-wide recurrent policy: latency.
        dict(name="scan_step_1", op="scan", T=1, N=1, D=256, dtype="fp32", fused=True, done=True, h0=True),
        # One control step of the 65,536-env rollout, 256 wide.
        dict(name="scan_step_65536", op="scan", T=1, N=65536, D=256, dtype="bf16", fused=True, done=True, h0=True),
        # Training pass over 128 steps of 4,096 envs, gate and value halves of one projection.
        dict(name="scan_4096x128", op="scan", T=128, N=4096, D=256, dtype="bf16", fused=True, done=True, h0=True),
        # One long log of a vehicle, odd length, a width of no vector's multiple.
        dict(name="scan_long", op="scan", T=65521, N=1, D=250, dtype="fp32", fused=False, done=False, h0=False),
        # Gradient of the training pass.
        dict(name="scan_back_4096x128", op="scan_back", T=128, N=4096, D=256, dtype="bf16", fused=True, done=True, h0=True),
        # Gradient over a few long logs with episode ends.
        dict(name="scan_back_long", op="scan_back", T=8192, N=5, D=100, dtype="fp16", fused=False, done=True, h0=True),
        # Layer norm and ReLU of a critic (one group, one position) over a 65,536-sample minibatch.
        dict(name="norm_rows_65536", op="norm", B=65536, S=1, C=256, G=1, act="relu", dtype="bf16", pad=0),
        # The same over an off-policy minibatch of 256 samples, nine groups of ten channels: latency, odd sizes.
        dict(name="norm_rows_256", op="norm", B=256, S=1, C=90, G=9, act="tanh", dtype="fp32", pad=0),
        # Group norm over whole sequences of features, statistics over 4,096 steps.
        dict(name="norm_seq_64", op="norm", B=64, S=4096, C=256, G=32, act="silu", dtype="bf16", pad=0),
        # Residual dropout of a 65,536-sample minibatch, and its gradient.
        dict(name="dropout_rows_65536", op="dropout", T=1, N=65536, D=256, p=0.1, dtype="bf16", shared=False, residual=True, pad=0),
        # One mask for a sequence's whole length (recurrent networks), odd sizes, a slice of a wider array.
        dict(name="dropout_shared", op="dropout", T=128, N=513, D=257, p=0.25, dtype="fp32", shared=True, residual=False, pad=7),
        # Off-policy minibatch of 256 samples: latency.
        dict(name="dropout_rows_256", op="dropout", T=1, N=256, D=256, p=0.01, dtype="fp32", shared=False, residual=False, pad=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["scan", "scan", "scan_back", "norm", "norm", "dropout"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    most = 60_000_000 if dtype != "fp32" else 30_000_000
    if op in ("scan", "scan_back"):
        T, N, D = _log(rng, 1, 65536), _log(rng, 1, 65536), _log(rng, 1, 1024)
        if rng.random() < 0.6:          # widths are mostly round
            D = max(8, D // 8 * 8)
        N = max(1, min(N, most // D))
        T = max(1, min(T, most // (N * D)))
        return dict(op=op, T=T, N=N, D=D, dtype=dtype, fused=rng.random() < 0.5, done=rng.random() < 0.7,
                    h0=rng.random() < 0.7)
    if op == "norm":
        G = rng.choice([1, 1, 2, 3, 4, 8, 9, 16, 32])
        C = G * _log(rng, 1, max(1, 1024 // G))
        if rng.random() < 0.6:
            C = max(1, C // G // 8) * 8 * G
        B = _log(rng, 1, 65536)
        S = 1 if rng.random() < 0.4 else _log(rng, 1, 16384)
        B = max(1, min(B, most // C))
        S = max(1, min(S, most // (B * C)))
        if C // G * S == 1:             # a group of one value has no spread to normalise
            S = 2
        # relu's slope jumps at 0: in 32 bits an element there follows the last bit of the statistics
        act = rng.choice(["none", "silu", "tanh"] if dtype == "fp32" else ["none", "relu", "silu", "tanh"])
        return dict(op=op, B=B, S=S, C=C, G=G, act=act, dtype=dtype, pad=rng.choice([0, 0, 0, 3, 8]))
    T, N, D = _log(rng, 1, 512), _log(rng, 1, 65536), _log(rng, 1, 1024)
    N = max(1, min(N, most // D))
    T = max(1, min(T, most // (N * D)))
    return dict(op=op, T=T, N=N, D=D, p=rng.choice([0.0, 0.01, 0.1, 0.25, 0.5, 0.9]), dtype=dtype,
                shared=rng.random() < 0.5, residual=rng.random() < 0.5, pad=rng.choice([0, 0, 0, 3, 8]))


# ------------------------------------------------------------------ inputs
def _normal(g, shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(shape, device="cuda", generator=g) * scale + shift).to(dtype)


def _padded(g, shape, pad, dtype, scale=1.0, shift=0.0):
    """Channels of a wider array: the last axis contiguous, rows `pad` elements further apart."""
    x = _normal(g, (*shape[:-1], shape[-1] + pad), dtype, scale, shift)
    return x[..., :shape[-1]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]
    st = dict(case=case)
    op = case["op"]
    if op in ("scan", "scan_back"):
        T, N, D = case["T"], case["N"], case["D"]
        shape = (T, N, D)

        def pair(f_scale, f_shift):     # gate and value: halves of one array, or two arrays
            if not case["fused"]:
                return _normal(g, shape, dt, f_scale, f_shift), _normal(g, shape, dt)
            z = _normal(g, (T, N, 2 * D), dt)
            z[..., :D].mul_(f_scale).add_(f_shift)
            return z[..., :D], z[..., D:]
        st["f"], st["v"] = pair(1.5, 2.0)      # gates that remember some ten steps, some channels for hundreds
        st["done"] = st["done_prev"] = st["h0"] = None
        if case["done"]:
            st["done"] = (torch.rand((T, N), device="cuda", generator=g) < 0.005).to(torch.uint8)
            st["done_prev"] = (torch.rand((N,), device="cuda", generator=g) < 0.1).to(torch.uint8)
        if case["h0"]:
            st["h0"] = _normal(g, (N, D), torch.float32, 0.5)
        if op == "scan":
            st["y"] = torch.empty(shape, device="cuda", dtype=dt)
            st["hT"] = torch.empty((N, D), device="cuda")
        else:
            st["y"] = _plain_scan(st)[0]        # the forward's output, as stored
            st["dy"] = _normal(g, shape, dt, 0.1)
            st["dhT"] = _normal(g, (N, D), torch.float32, 0.1)
            if case["fused"]:
                z = torch.empty((T, N, 2 * D), device="cuda", dtype=dt)
                st["df"], st["dv"] = z[..., :D], z[..., D:]
            else:
                st["df"], st["dv"] = (torch.empty(shape, device="cuda", dtype=dt) for _ in range(2))
            st["dh0"] = torch.empty((N, D), device="cuda")
    elif op == "norm":
        B, S, C = case["B"], case["S"], case["C"]
        st["x"] = _padded(g, (B, S, C), case["pad"], dt, 1.5, 0.3)
        st["dy"] = _padded(g, (B, S, C), case["pad"], dt, 0.1)
        st["gamma"] = _normal(g, (C,), torch.float32, 0.2, 1.0)
        st["beta"] = _normal(g, (C,), torch.float32, 0.2)
        st["y"], st["dx"] = (torch.empty((B, S, C), device="cuda", dtype=dt) for _ in range(2))
        st["mean"], st["rstd"] = (torch.empty((B, case["G"]), device="cuda") for _ in range(2))
        st["dgamma"], st["dbeta"] = (torch.empty((C,), device="cuda") for _ in range(2))
    else:
        shape = (case["T"], case["N"], case["D"])
        st["x"] = _padded(g, shape, case["pad"], dt)
        st["dy"] = _padded(g, shape, case["pad"], dt, 0.1)
        st["residual"] = _padded(g, shape, case["pad"], dt) if case["residual"] else None
        st["seed"], st["draw"] = 0x9E3779B97F4A7C15 ^ seed, 1 + seed % 1000
        st["y"], st["dx"] = (torch.empty(shape, device="cuda", dtype=dt) for _ in range(2))
    return st


# ------------------------------------------------------------------ plain forms
def _ended(st, T, N):
    """[T, N, 1]: whether an episode ended before step t."""
    if st["done"] is None:
        return torch.zeros((T, N, 1), dtype=torch.bool, device="cuda")
    return torch.cat([st["done_prev"][None], st["done"][:-1]]).bool()[..., None]


def _scan(A, X):
    """h_t = A_t h_{t-1} + X_t along the first axis (h before it 0) by doubling: after a round each element holds its
    last 2, 4, 8, ... steps.  Exact zeros of A cut the past off."""
    s = 1
    while s < X.shape[0]:
        X = torch.cat([X[:s], torch.where(A[s:] == 0, X[s:], A[s:] * X[:-s] + X[s:])])
        A = torch.cat([A[:s], A[s:] * A[:-s]])
        s *= 2
    return X


def _plain_scan(st):
    f, v = st["f"].float(), st["v"].float()
    T, N, D = f.shape
    ended = _ended(st, T, N)
    a = torch.sigmoid(f)
    X = torch.sigmoid(-f) * v
    if st["h0"] is not None:
        X[0] += torch.where(ended[0], 0.0, a[0] * st["h0"])
    h = _scan(torch.where(ended, 0.0, a), X)
    return h.to(st["f"].dtype), h[-1].clone()


def _plain_scan_back(st):
    f, v, y, dy = (st[k].float() for k in ("f", "v", "y", "dy"))
    T, N, D = f.shape
    ended = _ended(st, T, N)
    a, b = torch.sigmoid(f), torch.sigmoid(-f)
    h0 = st["h0"] if st["h0"] is not None else torch.zeros((N, D), device="cuda")
    c = torch.where(ended, 0.0, torch.cat([h0[None], y[:-1]]))
    keep = torch.where(ended, 0.0, a)
    X = dy.clone()
    X[-1] += st["dhT"]
    # d_t = dy_t + keep_{t+1} d_{t+1}, from the last step to the first
    A = torch.cat([keep[1:], torch.zeros_like(keep[:1])])
    d = _scan(A.flip(0), X.flip(0)).flip(0)
    t = st["f"].dtype
    return (a * b * (c - v) * d).to(t), (b * d).to(t), keep[0] * d[0]


def _act(u, act):
    """act(u) and its derivative."""
    if act == "relu":
        return torch.clamp_min(u, 0.0), (u > 0).float()
    if act == "silu":
        s = torch.sigmoid(u)
        return u * s, s * (1 + u * (1 - s))
    if act == "tanh":
        t = torch.tanh(u)
        return t, 1 - t * t
    return u, torch.ones_like(u)


EPS = 1e-5


def _plain_norm(st):
    x, dy = st["x"].float(), st["dy"].float()
    B, S, C = x.shape
    G = st["case"]["G"]
    xg = x.reshape(B, S, G, C // G)
    mean = xg.mean(dim=(1, 3), keepdim=True)
    var = ((xg - mean) ** 2).mean(dim=(1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(var + EPS)
    xh = ((xg - mean) * rstd).view(B, S, C)
    y, slope = _act(xh * st["gamma"] + st["beta"], st["case"]["act"])
    dz = dy * slope
    dbeta, dgamma = dz.sum(dim=(0, 1)), (dz * xh).sum(dim=(0, 1))
    w = (dz * st["gamma"]).view(B, S, G, C // G)
    xh = xh.view(B, S, G, C // G)
    m1, m2 = w.mean(dim=(1, 3), keepdim=True), (w * xh).mean(dim=(1, 3), keepdim=True)
    dx = (rstd * (w - m1 - xh * m2)).view(B, S, C)
    t = st["x"].dtype
    return y.to(t), mean.view(B, G), rstd.view(B, G), dx.to(t), dgamma, dbeta


def _philox(blocks, key0, key1, draw):
    """Philox4x32-10 words at counters (block low, block high, draw low, draw high), as [n, 4] integers."""
    m = 0xFFFFFFFF
    c0, c1 = blocks & m, blocks >> 32
    c2, c3 = torch.full_like(c0, draw & m), torch.full_like(c0, draw >> 32)
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57      # 64-bit products, the sign bit used as a digit
        c0, c1, c2, c3 = (p1 >> 32 & m) ^ c1 ^ key0, p1 & m, (p0 >> 32 & m) ^ c3 ^ key1, p0 & m
        key0, key1 = key0 + 0x9E3779B9 & m, key1 + 0xBB67AE85 & m
    return torch.stack([c0, c1, c2, c3], dim=1)


def _keep(n, p, seed, draw):
    """[n] of 0 (dropped) and 1 / (1 - p), p in steps of 2^-16."""
    thr = round(p * 65536)
    w = _philox(torch.arange((n + 7) // 8, device="cuda"), seed & 0xFFFFFFFF, seed >> 32, draw)
    u = torch.stack([w & 0xFFFF, w >> 16], dim=2).view(-1)[:n]
    return torch.where(u < thr, 0.0, 65536 / (65536 - thr))


def _plain_dropout(st):
    case = st["case"]
    T, N, D = case["T"], case["N"], case["D"]
    shape = (1, N, D) if case["shared"] else (T, N, D)
    k = _keep(math.prod(shape), case["p"], st["seed"], st["draw"]).view(shape)
    y = st["x"].float() * k
    if st["residual"] is not None:
        y = y + st["residual"].float()
    t = st["x"].dtype
    return y.to(t), (st["dy"].float() * k).to(t)


# ------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return {"scan": _plain_scan, "scan_back": _plain_scan_back, "norm": _plain_norm,
                "dropout": _plain_dropout}[op](st)
    from paper_2512_13359_gb300 import nets
    if op == "scan":
        return nets.gate_scan(st["f"], st["v"], st["h0"], done=st["done"], done_prev=st["done_prev"], y=st["y"],
                              hT=st["hT"])
    if op == "scan_back":
        return nets.gate_scan_backward(st["f"], st["v"], st["y"], st["dy"], st["h0"], done=st["done"],
                                       done_prev=st["done_prev"], dhT=st["dhT"], df=st["df"], dv=st["dv"],
                                       dh0=st["dh0"])
    if op == "norm":
        y, mean, rstd = nets.group_norm(st["x"], case["G"], st["gamma"], st["beta"], eps=EPS, act=case["act"],
                                        y=st["y"], mean=st["mean"], rstd=st["rstd"])
        dx, dgamma, dbeta = nets.group_norm_backward(st["x"], case["G"], st["gamma"], st["beta"], mean, rstd,
                                                     st["dy"], act=case["act"], dx=st["dx"], dgamma=st["dgamma"],
                                                     dbeta=st["dbeta"])
        return y, mean, rstd, dx, dgamma, dbeta
    y = nets.dropout(st["x"], case["p"], st["seed"], st["draw"], residual=st["residual"], shared=case["shared"],
                     y=st["y"])
    return y, nets.dropout(st["dy"], case["p"], st["seed"], st["draw"], shared=case["shared"], y=st["dx"])


def work(case):
    """Bytes: each input once, each output once.  Operations: of the formulas, an exponential or a division as one."""
    op, z = case["op"], SIZE[case["dtype"]]
    if op in ("scan", "scan_back"):
        n, m = case["T"] * case["N"] * case["D"], case["N"] * case["D"]
        ends = case["T"] * case["N"] if case["done"] else 0
        states = (1 + case["h0"]) if op == "scan" else (2 + case["h0"])     # hT, h0; dhT, dh0, h0
        return {"bytes": n * z * (3 if op == "scan" else 6) + ends + 4 * m * states,
                "flops": n * (8 if op == "scan" else 13)}
    if op == "norm":
        n = case["B"] * case["S"] * case["C"]
        return {"bytes": 4 * n * z + 8 * case["B"] * case["G"] + 16 * case["C"], "flops": 30 * n}
    n = case["T"] * case["N"] * case["D"]
    return {"bytes": n * z * (5 if case["residual"] else 4), "flops": n * (3 if case["residual"] else 2)}


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"scan": _exact_scan, "scan_back": _exact_scan_back, "norm": _exact_norm, "dropout": _exact_dropout}[
        case["op"]](st)


def _exact_ended(st, t):
    return None if st["done"] is None else (st["done_prev"] if t == 0 else st["done"][t - 1]).ne(0)[:, None]


def _exact_scan(st):
    T, N, D = st["f"].shape
    h = torch.zeros((N, D), dtype=torch.float64, device="cuda") if st["h0"] is None else st["h0"].double()
    y = torch.empty((T, N, D), dtype=torch.float64, device="cuda")
    for t in range(T):
        e = _exact_ended(st, t)
        h = h if e is None else h.masked_fill(e, 0.0)
        g = torch.sigmoid(st["f"][t].double())
        h = torch.add(g * (h - st["v"][t]), st["v"][t], out=y[t])
    return y, h.clone()


def _exact_scan_back(st):
    T, N, D = st["f"].shape
    g = st["dhT"].double()
    df, dv = (torch.empty((T, N, D), dtype=torch.float64, device="cuda") for _ in range(2))
    for t in reversed(range(T)):
        e = _exact_ended(st, t)
        before = st["y"][t - 1].double() if t else (st["h0"].double() if st["h0"] is not None else torch.zeros_like(g))
        before = before if e is None else before.masked_fill(e, 0.0)
        s = torch.sigmoid(st["f"][t].double())
        d = g + st["dy"][t]
        dv[t] = d - s * d
        df[t] = d * (before - st["v"][t]) * (s - s * s)
        g = s * d if e is None else (s * d).masked_fill(e, 0.0)
    return df, dv, g


def _exact_norm(st):
    case = st["case"]
    B, S, C = st["x"].shape
    x, gamma, beta = (st[k].double().detach().requires_grad_() for k in ("x", "gamma", "beta"))
    xg = x.reshape(B, S, case["G"], C // case["G"])
    var, mean = torch.var_mean(xg, dim=(1, 3), unbiased=False, keepdim=True)
    rstd = (var + EPS) ** -0.5
    u = ((xg - mean) * rstd).reshape(B, S, C) * gamma + beta
    y = {"none": lambda q: q, "relu": torch.relu, "silu": lambda q: q / (1 + torch.exp(-q)), "tanh": torch.tanh}[
        case["act"]](u)
    dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), st["dy"].double())
    G = case["G"]
    return y.detach(), mean.detach().reshape(B, G), rstd.detach().reshape(B, G), dx, dgamma, dbeta


def _exact_dropout(st):
    case = st["case"]
    shape = (1 if case["shared"] else case["T"], case["N"], case["D"])
    n = math.prod(shape)
    block = np.arange((n + 7) // 8, dtype=np.uint64)
    u32 = np.uint64(0xFFFFFFFF)
    c = [block & u32, block >> np.uint64(32), np.full_like(block, st["draw"] & 0xFFFFFFFF),
         np.full_like(block, st["draw"] >> 32)]
    k = [st["seed"] & 0xFFFFFFFF, st["seed"] >> 32]
    for r in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        ka, kb = (np.uint64((k[i] + r * w) & 0xFFFFFFFF) for i, w in ((0, 0x9E3779B9), (1, 0xBB67AE85)))
        c = [(b >> np.uint64(32)) ^ c[1] ^ ka, b & u32, (a >> np.uint64(32)) ^ c[3] ^ kb, a & u32]
    bits = np.stack(c, axis=1).astype("<u4").view("<u2").reshape(-1)[:n]
    thr = int(math.floor(case["p"] * 65536 + 0.5))
    keep = torch.from_numpy((bits >= thr).astype(np.float64)).cuda().view(shape) * (65536.0 / (65536 - thr))
    y = st["x"].double() * keep
    if st["residual"] is not None:
        y = y + st["residual"].double()
    return y, st["dy"].double() * keep
