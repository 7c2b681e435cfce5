"""The state space memory (causal_conv, select_scan) and the orthogonalised update on a GPU against the 64-bit reference
(state_ref.py), whose bounds come with it: types, odd and ragged sizes, lengths from none to 20,000, strides, groups, episode
ends everywhere, infinities and NaN behind them, states in place, other streams, CUDA graphs, repeated calls bit for bit,
refusals, and the three together as a layer that is trained."""
import numpy as np
import pytest

import nets_ref
import state_ref as R
from parity_util import need_gpu
from test_gpu_nets import _np, _rows, _within

pytestmark = pytest.mark.gpu

DT = ("fp32", "bf16", "fp16")


def _t():
    torch = need_gpu()
    from paper_2512_13359_gb300 import nets
    return torch, nets, {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _nn(x):
    return None if x is None else _np(x)


def _ends(torch, T, N, ends, g):
    if ends is None:
        return None, None
    return ((torch.rand((T, N), device="cuda", generator=g) < ends).to(torch.uint8),
            (torch.rand((N,), device="cuda", generator=g) < max(ends, 0.3)).to(torch.uint8))


# ------------------------------------------------------------ convolution
def _check_conv(T, N, D, K, dt, layout="flat", ends=0.1, seed=0, state=True, bias=True, act="silu"):
    torch, nets, types = _t()
    t = types[dt]
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(s, device="cuda", generator=g)   # noqa: E731
    x = _rows(torch, (T, N, D), t, layout, g)
    w, b = rn(K, D) * K ** -0.5, rn(D) * 0.3 if bias else None
    st = rn(K - 1, N, D).to(t) if state else None
    done, prev = _ends(torch, T, N, ends, g)
    b0 = np.zeros(D) if b is None else _np(b)
    y, new = nets.causal_conv(x, w, b, st, done=done, done_prev=prev, act=act, y=_rows(torch, (T, N, D), t, layout, g))
    ry, rn_, Ey = R.conv(_np(x), _np(w), b0, _nn(st), _nn(done), _nn(prev), act)
    _within(y, ry, Ey, dt)
    assert np.array_equal(_np(new), rn_)
    dy, dn = _rows(torch, (T, N, D), t, layout, g, 0.3), rn(K - 1, N, D).to(t) if state else None
    got = nets.causal_conv_backward(x, w, b, dy, st, done=done, done_prev=prev, act=act, dnew_state=dn,
                                    dx=_rows(torch, (T, N, D), t, layout, g))
    r = R.conv_backward(_np(x), _np(w), b0, _np(dy), _nn(st), _nn(done), _nn(prev), _nn(dn), act)
    for q, ref, E, kind in zip(got, r[:4], r[4:], (dt, "fp32", "fp32", dt)):
        _within(q, ref, E, kind)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,N,D,K", [(1, 1, 256, 4), (1, 70, 40, 4), (2, 3, 5, 4), (7, 33, 12, 3), (8, 5, 64, 1), (33, 4, 100, 2),
                                     (129, 2, 250, 4), (300, 9, 17, 5), (1000, 1, 8, 8), (57, 1, 1, 6), (9, 300, 24, 7), (3, 2, 2100, 4)])
def test_conv(T, N, D, K, dt):
    _check_conv(T, N, D, K, dt, seed=T)


@pytest.mark.parametrize("layout", ["odd", "pad", "half", "swap"])
@pytest.mark.parametrize("T,N,D,K,dt", [(20, 6, 24, 4, "bf16"), (20, 6, 24, 4, "fp32"), (700, 3, 16, 3, "fp16"), (40, 2, 33, 8, "bf16")])
def test_conv_strides(T, N, D, K, dt, layout):
    _check_conv(T, N, D, K, dt, layout, seed=5)


@pytest.mark.parametrize("ends", [None, 0.0, 0.6, 1.0])
@pytest.mark.parametrize("T,N,D,K", [(40, 9, 32, 4), (500, 2, 24, 8), (1, 4, 8, 4), (2, 4, 8, 8)])
def test_conv_ends(T, N, D, K, ends):
    _check_conv(T, N, D, K, "fp32", ends=ends, seed=6, state=ends != 0.6, bias=ends != 0.0, act="none" if ends == 1.0 else "silu")


def test_conv_long():
    _check_conv(20011, 1, 6, 4, "bf16", ends=0.001, seed=7)
    _check_conv(9001, 2, 8, 5, "fp32", ends=0.001, seed=8)


def test_conv_steps_in_place_are_one_pass():
    torch, nets, _ = _t()
    g = torch.Generator(device="cuda").manual_seed(1)
    T, N, D, K = 12, 5, 24, 4
    x, w = torch.randn(T, N, D, device="cuda", generator=g), torch.randn(K, D, device="cuda", generator=g)
    done, prev = _ends(torch, T, N, 0.2, g)
    y, new = nets.causal_conv(x, w, None, None, done=done, done_prev=prev)
    for step in (1, 2, 5):
        st, p, parts = torch.zeros(K - 1, N, D, device="cuda"), prev, []
        for t in range(0, T, step):
            s = slice(t, min(T, t + step))
            yt, out = nets.causal_conv(x[s], w, None, st, done=done[s], done_prev=p, new_state=st)
            assert out is st
            p = done[s][-1]
            parts.append(yt)
        assert torch.equal(torch.cat(parts), y) and torch.equal(st, new)


def test_conv_without_steps_or_envs():
    torch, nets, _ = _t()
    st, w = torch.randn(3, 4, 8, device="cuda"), torch.randn(4, 8, device="cuda")
    z = torch.empty(0, 4, 8, device="cuda")
    y, new = nets.causal_conv(z, w, None, st)
    assert y.numel() == 0 and torch.equal(new, st)
    assert torch.equal(nets.causal_conv(z, w)[1], torch.zeros_like(st))
    _, dw, db, ds = nets.causal_conv_backward(z, w, None, z, st, dnew_state=2 * st)
    assert torch.equal(ds, 2 * st) and not dw.any() and not db.any()
    z = torch.empty(5, 0, 8, device="cuda")
    _, dw, db, _ = nets.causal_conv_backward(z, w, None, z)
    assert not dw.any() and not db.any()


# ------------------------------------------------------------ scan
def _scan_args(torch, t, T, N, D, S, G, layout, ends, seed, gate=True, h0=True, extra=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(s, device="cuda", generator=g)   # noqa: E731
    rows = lambda k, sc=1.0: _rows(torch, (T, N, k), t, layout, g, sc)          # noqa: E731
    a = dict(x=rows(D), dt=rows(D, 0.5), B=rows(G * S), C=rows(G * S), A=-torch.exp(rn(D, S)))
    opt = dict(skip=rn(D) if extra else None, dt_bias=rn(D) - 1.5 if extra else None, gate=rows(D) if gate else None)
    opt["done"], opt["done_prev"] = _ends(torch, T, N, ends, g)
    return g, a, opt, rn(N, D, S) if h0 else None


def _check_scan(T, N, D, S, G, dt, layout="flat", ends=0.1, seed=0, gate=True, h0=True, extra=True):
    torch, nets, types = _t()
    g, a, opt, h0 = _scan_args(torch, types[dt], T, N, D, S, G, layout, ends, seed, gate, h0, extra)
    y = _rows(torch, (T, N, D), types[dt], layout, g)
    y, hT, kept = nets.select_scan(**a, **opt, h0=h0, kept=True, y=y)
    q = R.Scan(*(_nn(v) for v in (a["x"], a["dt"], a["A"], a["B"], a["C"], opt["skip"], opt["dt_bias"], opt["gate"], h0,
                                  opt["done"], opt["done_prev"])))
    _within(y, q.y, q.Ey, dt)
    _within(hT, q.hT, q.EhT)
    _within(kept, np.stack(q.kept), np.stack(q.Ekept))
    plain = nets.select_scan(**a, **opt, h0=h0)
    assert torch.equal(plain[0], y) and plain[2] is None         # kept or not, the same pass
    dy = _rows(torch, (T, N, D), types[dt], layout, g, 0.5)
    dhT = torch.randn(N, D, S, device="cuda", generator=g) if h0 is not None else None
    names = ("dx", "ddt", "dA", "dB", "dC", "dskip", "ddt_bias", "dgate", "dh0")
    outs = {k: _rows(torch, (T, N, G * S if k in ("dB", "dC") else D), types[dt], layout, g) for k in ("dx", "ddt", "dB", "dC")}
    got = dict(zip(names, nets.select_scan_backward(*(a[k] for k in ("x", "dt", "A", "B", "C")), kept, dy, **opt, dhT=dhT, **outs)))
    ref = q.backward(_np(dy), _nn(dhT))
    for k in names:
        if k == "dgate" and not gate:
            assert got[k] is None
            continue
        _within(got[k], *ref[k], dt if got[k].dtype is not torch.float32 else "fp32")


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,N,D,S,G", [(1, 1, 64, 16, 1), (1, 70, 40, 8, 1), (2, 3, 5, 4, 1), (7, 33, 12, 13, 2), (16, 5, 64, 16, 1),
                                       (17, 4, 100, 16, 4), (33, 2, 250, 13, 1), (50, 9, 17, 1, 1), (40, 2, 24, 32, 2), (20, 3, 10, 64, 1),
                                       (19, 2, 7, 128, 1), (18, 2, 600, 16, 1), (21, 1, 300, 3, 1)])
def test_scan(T, N, D, S, G, dt):
    _check_scan(T, N, D, S, G, dt, seed=T)


@pytest.mark.parametrize("layout", ["odd", "pad", "half", "swap"])
@pytest.mark.parametrize("T,N,D,S,G,dt", [(20, 6, 24, 16, 1, "bf16"), (20, 6, 24, 8, 2, "fp32"), (300, 2, 16, 16, 1, "fp16")])
def test_scan_strides(T, N, D, S, G, dt, layout):
    _check_scan(T, N, D, S, G, dt, layout, seed=5)


@pytest.mark.parametrize("ends", [None, 0.0, 0.6, 1.0])
@pytest.mark.parametrize("T,N,D,S", [(40, 5, 32, 16), (400, 2, 24, 4), (1, 4, 8, 16)])
def test_scan_ends(T, N, D, S, ends):
    _check_scan(T, N, D, S, 1, "fp32", ends=ends, seed=6, h0=ends != 0.6, gate=ends != 0.0, extra=ends != 1.0)


@pytest.mark.parametrize("T,N,D,S,G,dt", [(3001, 1, 20, 13, 1, "fp32"), (2049, 2, 12, 8, 2, "bf16"), (1500, 1, 40, 16, 1, "fp16"),
                                          (128, 1, 3, 4, 1, "fp32"), (129, 1, 9, 1, 1, "bf16"), (1000, 3, 5, 40, 1, "fp32")])
def test_scan_long(T, N, D, S, G, dt):
    _check_scan(T, N, D, S, G, dt, ends=0.002, seed=7)


@pytest.mark.parametrize("T,N,D,S,G,dt,layout", [(19, 1900, 40, 16, 1, "bf16", "flat"), (5, 950, 96, 13, 1, "fp16", "half"), (6, 2000, 6, 8, 1, "fp32", "flat"),
                                                 (18, 950, 12, 3, 2, "bf16", "pad"), (4, 2000, 34, 10, 1, "fp32", "odd")])
def test_scan_of_many_envs(T, N, D, S, G, dt, layout):
    """Enough warps for two channels a lane, or not aligned for it."""
    _check_scan(T, N, D, S, G, dt, layout, seed=13)


@pytest.mark.parametrize("T,N,D,S,G,dt,layout", [(37, 50, 8, 16, 1, "bf16", "flat"), (40, 7, 16, 16, 2, "fp16", "half"), (19, 900, 2, 13, 1, "fp32", "odd"),
                                                 (33, 6, 12, 4, 3, "bf16", "swap"), (700, 2, 6, 8, 1, "fp32", "flat"), (900, 1, 7, 16, 1, "bf16", "pad"),
                                                 (16, 3, 32, 8, 4, "fp32", "flat"), (130, 5, 1, 1, 1, "fp16", "flat"), (65, 601, 8, 5, 1, "fp32", "pad")])
def test_scan_of_narrow_groups(T, N, D, S, G, dt, layout):
    """Four rows a warp, the last of them without rows for all."""
    _check_scan(T, N, D, S, G, dt, layout, ends=0.05, seed=14)


def _against_formulas(a, h0, dy=None):
    """select_scan of inputs without ends, gate or bias, and its gradients, against the 64-bit reference."""
    torch, nets, _ = _t()
    y, hT, kept = nets.select_scan(**a, h0=h0, kept=True)
    q = R.Scan(*(_np(a[k]) for k in ("x", "dt", "A", "B", "C")), None, None, None, _nn(h0), None, None)
    _within(y, q.y, q.Ey)
    _within(hT, q.hT, q.EhT)
    if dy is not None:
        names = ("dx", "ddt", "dA", "dB", "dC", "dskip", "ddt_bias", "dgate", "dh0")
        got, ref = dict(zip(names, nets.select_scan_backward(*(a[k] for k in ("x", "dt", "A", "B", "C")), kept, dy))), q.backward(_np(dy), None)
        for k in ref:
            _within(got[k], *ref[k])
    return hT


@pytest.mark.parametrize("octave", [4, 5, 6])
def test_scan_decays_are_not_off_to_one_side(octave):
    """4,096 decays 2^t, t between -2^-octave and half of that, of constant inputs: a state is off by the error of its decay
    times the mean age of what it holds.  Over all t of these octaves the unit's exponential is 0.29 to 0.45 units of 2^-24 low,
    and 0.26 of them are given back: 0.19 on average at most, and 0.01 for 4,096 decays that are 0.7 off at random.  e and its
    products, 2 units once: a state that has forgotten its start is 1 / |A|, whatever e is."""
    torch, nets, _ = _t()
    T, D, S = 512, 256, 16
    g = torch.Generator(device="cuda").manual_seed(octave)
    one = lambda k: torch.ones(T, 1, k, device="cuda")           # noqa: E731
    A = -(2.0 ** -octave) * (0.5 + 0.5 * torch.rand(D, S, device="cuda", generator=g))      # e log2(e) = 1 at dt = 0
    _, hT, _ = nets.select_scan(one(D), torch.zeros(T, 1, D, device="cuda"), A, one(S), one(S))
    e, a = np.log(2.0), np.exp(np.log(2.0) * _np(A))
    j = np.arange(T)[:, None, None]
    weight = a ** j
    age = (j * weight).sum(0) / weight.sum(0)
    off = (_np(hT)[0] / (e * weight.sum(0)) - 1) / R.U
    assert abs((off / age).mean()) <= 0.2 + 2 / age.min()


@pytest.mark.parametrize("T", [1, 40, 700])
def test_scan_of_states_that_stay(T):
    """Where a step size or a rate is 0 a state passes bit for bit, and so does its gradient."""
    torch, nets, types = _t()
    D, S = 40, 16
    g, a, opt, h0 = _scan_args(torch, types["fp32"], T, 2, D, S, 1, "flat", None, 2, gate=False, extra=False)
    dhT, zero = torch.randn(2, D, S, device="cuda", generator=g), torch.zeros(T, 2, D, device="cuda")
    still = dict(a, x=zero, dt=torch.full_like(zero, -float("inf")))
    flat = dict(a, x=zero, A=torch.zeros(D, S, device="cuda"))
    for q in (still, flat):
        _, hT, kept = nets.select_scan(**q, h0=h0, kept=True)
        assert torch.equal(hT, h0) and torch.equal(kept, h0.expand_as(kept))
        grads = nets.select_scan_backward(*(q[k] for k in ("x", "dt", "A", "B", "C")), kept, zero, dhT=dhT)
        assert torch.equal(grads[8], dhT)

@pytest.mark.parametrize("D,S", [(8, 4), (40, 16)])
@pytest.mark.parametrize("T", [1000, 20000])
def test_scan_of_growing_states(T, D, S):
    """A > 0: over a piece of a long sequence a state would grow past fp32's range, but it is 0 until the last steps (and its
    gradient from the first steps on)."""
    torch, nets, types = _t()
    g, a, _, _ = _scan_args(torch, types["fp32"], T, 1, D, S, 1, "flat", None, 3)
    a["A"], a["dt"] = 0.5 + 0.5 * torch.rand(D, S, device="cuda", generator=g), 1.0 + 0.1 * a["dt"]
    late, early = torch.zeros(2, T, 1, D, device="cuda")
    late[-20:], early[:20] = a["x"][-20:], a["x"][:20]
    hT = _against_formulas(dict(a, x=late), None)
    assert hT.abs().max() > 1e3
    _against_formulas(dict(a, x=torch.zeros_like(late)), None, early)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("T", [160, 1000])
def test_scan_of_states_that_pass_a_range_of_their_own(T, sign):
    """From 2^-100 up by 2^140, or from 2^100 down by as much, in the first piece of a sequence: in fp32's range at both ends."""
    torch, nets, types = _t()
    D, S = 8, 4
    g, a, _, _ = _scan_args(torch, types["fp32"], T, 1, D, S, 1, "flat", None, 5)
    a["dt"].fill_(-20.0)
    a["dt"][:60] = 1.0
    steps = 60 * np.log1p(np.e)                                   # the sum of the step sizes that count
    a["A"] = torch.full((D, S), sign * 140 * np.log(2.0) / steps, device="cuda")
    a["x"].zero_()
    h0 = torch.randn(1, D, S, device="cuda", generator=g) * 2.0 ** (-100 * sign)
    hT = _against_formulas(a, h0)
    assert (hT.double() / h0.double()).log2().sub(140 * sign).abs().max() < 0.1
    h0[0, 0] = float("inf")
    assert torch.isinf(nets.select_scan(**a, h0=h0)[1][0, 0]).all()


@pytest.mark.parametrize("T", [40, 20000])
def test_scan_of_a_constant_input_reaches_its_limit(T):
    """dt = 0, no bias: e = log 2; with B x = 1 the state goes to e / (1 - exp(e A)) times 1 minus exp(e A T), whatever the
    way through the steps."""
    torch, nets, _ = _t()
    D, S = 8, 4
    one = lambda k: torch.ones(T, 1, k, device="cuda")           # noqa: E731
    A = -torch.logspace(-4, 0.5, S, device="cuda").repeat(D, 1)
    y, hT, _ = nets.select_scan(one(D), torch.zeros(T, 1, D, device="cuda"), A, one(S), one(S))
    e, A64 = np.log(2.0), _np(A)
    want = e * (1 - np.exp(e * A64 * T)) / (1 - np.exp(e * A64))
    # each step: decay off by some 8 units, input by 16; over the memory of the state, 1 / (1 - a) steps
    tol = R.U * 32 / (1 - np.exp(e * A64))
    assert (np.abs(_np(hT)[0] / want - 1) <= np.minimum(tol, 32 * T * R.U)).all()
    assert np.abs(_np(y)[-1, 0] / want.sum(-1) - 1).max() <= 32 * T * R.U


def test_scan_steps_in_place_are_one_pass():
    torch, nets, types = _t()
    T, N, D, S = 40, 5, 24, 16
    g, a, opt, h0 = _scan_args(torch, types["fp32"], T, N, D, S, 1, "flat", 0.1, 3)
    y, hT, _ = nets.select_scan(**a, **opt, h0=h0)
    done, prev = opt.pop("done"), opt.pop("done_prev")
    gate = opt.pop("gate")
    for step in (1, 7, 16):
        h, p, parts = h0.clone(), prev, []
        for t in range(0, T, step):
            s = slice(t, min(T, t + step))
            part = {k: v if k == "A" else v[s] for k, v in a.items()}
            yt, out, _ = nets.select_scan(**part, **opt, gate=gate[s], h0=h, done=done[s], done_prev=p, hT=h)
            assert out is h
            p = done[s][-1]
            parts.append(yt)
        assert torch.equal(torch.cat(parts), y) and torch.equal(h, hT)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("G", [1, 2])
@pytest.mark.parametrize("S", [1, 3, 4, 8, 13, 16, 20, 24, 32, 40, 48, 56, 64, 72, 88, 96, 120, 128])
def test_single_steps_of_any_number_of_states(S, G, dt):
    """Against the formulas; rows that belong to nobody hold NaN; and two steps in place are a pass of two, bit for bit."""
    torch, nets, types = _t()
    t, N, D = types[dt], 37, 40
    g, a, opt, h0 = _scan_args(torch, t, 2, N, D, S, G, "flat", 0.2, S)
    for k in ("B", "C"):                                         # rows 16 apart, and one behind the last, aligned as before
        room = torch.full((2, N + 1, G * S + 16), float("nan"), device="cuda", dtype=t)
        room[:, :N, :G * S] = a[k]
        a[k] = room[:, :N, :G * S]
    first = {k: v if k == "A" else v[:1] for k, v in a.items()}
    gate, done, prev = opt.pop("gate"), opt.pop("done"), opt.pop("done_prev")
    y, h, kept = nets.select_scan(**first, **opt, gate=gate[:1], h0=h0, done_prev=prev, kept=True)
    q = R.Scan(*(_nn(v) for v in (first["x"], first["dt"], a["A"], first["B"], first["C"], opt["skip"], opt["dt_bias"], gate[:1], h0, None, prev)))
    _within(y, q.y, q.Ey, dt)
    _within(h, q.hT, q.EhT)
    assert torch.equal(kept[0], h0)
    want, hT, _ = nets.select_scan(**a, **opt, gate=gate, h0=h0, done=done, done_prev=prev)
    second = {k: v if k == "A" else v[1:] for k, v in a.items()}
    y2, out, _ = nets.select_scan(**second, **opt, gate=gate[1:], h0=h, done_prev=done[0], hT=h)
    assert out is h and torch.equal(y[0], want[0]) and torch.equal(y2[0], want[1]) and torch.equal(h, hT)


@pytest.mark.parametrize("N,D,S,G,dt,layout", [(5000, 12, 24, 1, "bf16", "flat"), (5000, 24, 40, 2, "fp32", "odd"), (3, 600, 48, 1, "fp16", "pad"),
                                               (1, 4, 120, 1, "fp32", "flat"), (2500, 16, 96, 4, "bf16", "half"), (7, 1, 24, 1, "fp16", "swap")])
def test_single_steps_of_padded_states(N, D, S, G, dt, layout):
    """More envs than warps walk side by side, odd strides, a single row; the states' gradients too."""
    _check_scan(1, N, D, S, G, dt, layout, ends=0.2, seed=S)


def test_scan_without_steps_or_envs():
    torch, nets, _ = _t()
    h0, A = torch.randn(3, 8, 4, device="cuda"), -torch.ones(8, 4, device="cuda")
    z, b = torch.empty(0, 3, 8, device="cuda"), torch.empty(0, 3, 4, device="cuda")
    y, hT, kept = nets.select_scan(z, z, A, b, b, h0=h0, kept=True)
    assert y.numel() == 0 and torch.equal(hT, h0) and kept.shape == (0, 3, 8, 4)
    out = nets.select_scan_backward(z, z, A, b, b, kept, z, dhT=2 * h0)
    assert torch.equal(out[-1], 2 * h0) and not out[2].any() and not out[5].any() and not out[6].any()
    z, b = torch.empty(5, 0, 8, device="cuda"), torch.empty(5, 0, 4, device="cuda")
    _, _, kept = nets.select_scan(z, z, A, b, b, kept=True)
    assert not nets.select_scan_backward(z, z, A, b, b, kept, z)[2].any()


def test_scan_without_channels():
    torch, nets, types = _t()
    for dt in DT:
        z, b = torch.empty(3, 2, 0, device="cuda", dtype=types[dt]), torch.ones(3, 2, 8, device="cuda", dtype=types[dt])
        A, dB, dC = torch.empty(0, 4, device="cuda"), torch.ones_like(b), torch.ones(3, 2, 16, device="cuda", dtype=types[dt])[..., 8:]
        y, _, kept = nets.select_scan(z, z, A, b, b, kept=True)
        nets.select_scan_backward(z, z, A, b, b, kept, y, dB=dB, dC=dC)
        assert not dB.any() and not dC.any()


@pytest.mark.parametrize("T", [6, 400])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_nothing_of_an_ended_episode_passes(T, bad):
    torch, nets, types = _t()
    N, D, S, K = 3, 16, 8, 4
    g, a, opt, h0 = _scan_args(torch, types["fp32"], T, N, D, S, 1, "flat", 0.0, 9)
    opt["done_prev"].zero_()
    opt["done"][T // 2, 1] = 1
    opt["done_prev"][2] = 1
    clean_h = h0.clone()
    clean_h[2] = 0
    want = nets.select_scan(**a, **opt, h0=clean_h, kept=True)
    dirty = {k: v.clone() for k, v in a.items()}
    dirty["x"][:T // 2 + 1, 1] = bad
    h0[2] = bad
    got = nets.select_scan(**dirty, **opt, h0=h0, kept=True)
    for y, z in zip(got[:2], want[:2]):
        assert torch.equal(y[..., 2, :] if y.dim() == 3 and y.shape[0] == T else y[2], z[..., 2, :] if z.dim() == 3 and z.shape[0] == T else z[2])
    assert torch.equal(got[0][T // 2 + 1:, 1], want[0][T // 2 + 1:, 1]) and torch.equal(got[1], want[1])
    dy = torch.randn(T, N, D, device="cuda", generator=g)
    grads = [nets.select_scan_backward(*(q[k] for k in ("x", "dt", "A", "B", "C")), kept, dy, **opt)
             for q, kept in ((dirty, got[2]), (a, want[2]))]
    for k in (0, 1, 3, 4, 7):                                    # gradients of the rows that see nothing of it
        assert torch.equal(grads[0][k][:, 2], grads[1][k][:, 2]) and torch.equal(grads[0][k][T // 2 + 1:, 1], grads[1][k][T // 2 + 1:, 1])
    assert not grads[0][8][2].any()
    w = torch.randn(K, D, device="cuda", generator=g)
    st = torch.randn(K - 1, N, D, device="cuda", generator=g)
    st[:, 2] = bad
    y, _ = nets.causal_conv(dirty["x"], w, None, st, done=opt["done"], done_prev=opt["done_prev"])
    z, _ = nets.causal_conv(a["x"], w, None, clean_h[0, 0, 0] * 0 + torch.where(torch.isfinite(st), st, 0.0), done=opt["done"],
                            done_prev=opt["done_prev"])
    assert torch.equal(y[:, 2], z[:, 2]) and torch.equal(y[T // 2 + 1:, 1], z[T // 2 + 1:, 1])


def test_offsets_past_32_bits():
    """A row of envs beyond 2^32 elements of the array, one step and three."""
    torch, nets, _ = _t()
    N, D, S = 70000, 8, 8
    wide = torch.zeros(N, 1, 66000, device="cuda", dtype=torch.bfloat16)         # 9.2 GB
    x = wide.transpose(0, 1)[..., :D]
    g = torch.Generator(device="cuda").manual_seed(2)
    x[0, -5:] = torch.randn(5, D, device="cuda", generator=g).to(torch.bfloat16)
    assert x.stride(1) * (N - 1) > 1 << 32
    w = torch.randn(4, D, device="cuda", generator=g)
    y, _ = nets.causal_conv(x, w)
    assert not y[0, :-5].any() and torch.equal(y[0, -5:], (w[3] * x[0, -5:].float()).to(torch.bfloat16))
    A, b = -torch.ones(D, S, device="cuda"), torch.ones(1, N, S, device="cuda", dtype=torch.bfloat16)
    z = torch.zeros(1, N, D, device="cuda", dtype=torch.bfloat16)
    y, hT, _ = nets.select_scan(x, z, A, b, b)
    want = np.log(2.0) * _np(x[0, -5:])
    assert not hT[:-5].any() and np.abs(_np(hT[-5:]) - want[..., None]).max() <= 16 * R.U * np.abs(want).max()


# ------------------------------------------------------------ update
def _check_ortho(L, M, N, dt, layout="flat", steps=5, seed=0, scale=1e-3, coef=(3.4445, -4.775, 2.0315), eps=1e-7):
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = _rows(torch, (L, M, N), types[dt], layout, g, scale)
    y = nets.orthogonalise(x, steps, coef=coef, eps=eps, y=_rows(torch, (L, M, N), types[dt], layout, g))
    got, x64 = _np(y), _np(x)
    assert np.isfinite(got).all()
    for i in range(L):
        ref, E = R.orthogonalise(x64[i], steps, coef, eps)
        bound = E + nets_ref.ROUND[dt] * (np.linalg.norm(ref) + E) + nets_ref.TINY[dt] * np.sqrt(M * N)
        assert np.linalg.norm(got[i] - ref) <= bound, (i, np.linalg.norm(got[i] - ref) / bound)
    return x, y


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("L,M,N", [(1, 1, 1), (2, 1, 9), (2, 9, 1), (3, 16, 16), (2, 100, 37), (2, 37, 100), (1, 128, 128), (1, 129, 257),
                                   (1, 300, 129), (5, 64, 64), (1, 256, 700), (1, 700, 256)])
def test_update(L, M, N, dt):
    _check_ortho(L, M, N, dt, seed=M)


@pytest.mark.parametrize("layout", ["odd", "pad", "half", "swap"])
@pytest.mark.parametrize("L,M,N,dt", [(3, 40, 24, "bf16"), (2, 24, 40, "fp32"), (2, 33, 130, "fp16")])
def test_update_strides(L, M, N, dt, layout):
    _check_ortho(L, M, N, dt, layout, seed=5)


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 9])
def test_update_steps(steps):
    _check_ortho(2, 50, 70, "fp32", steps=steps, seed=4)
    _check_ortho(2, 70, 50, "bf16", steps=steps, seed=4)


def test_update_coefficients():
    _check_ortho(2, 30, 40, "fp32", steps=8, coef=(1.5, -0.5, 0.0))          # to the nearest isometry
    x, y = _check_ortho(1, 30, 40, "fp32", steps=30, coef=(1.5, -0.5, 0.0))
    s = np.linalg.svd(_np(y)[0], compute_uv=False)
    assert np.abs(s - 1).max() < 1e-5
    _check_ortho(2, 30, 40, "fp32", steps=3, coef=(-2.0, 1.5, -0.5))


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 1e15, 1e30])
def test_update_whatever_the_scale(scale):
    """Norms whose squares are out of fp32's range, either way."""
    _check_ortho(2, 20, 30, "fp32", scale=scale, eps=0.0, seed=8)
    if scale == 1e30:
        _check_ortho(1, 20, 30, "bf16", scale=scale, seed=8)


@pytest.mark.parametrize("L,M,N,dt,scale,steps", [(2, 64, 80, "fp32", 5e37, 5), (1, 300, 500, "fp32", 5e37, 0), (2, 300, 500, "bf16", 5e37, 2),
                                                  (2, 64, 80, "fp32", 1e16, 1), (2, 64, 80, "fp32", 1e-14, 1), (2, 100, 70, "fp32", 1e-42, 5),
                                                  (2, 100, 70, "fp32", 1e-42, 0), (1, 40, 1000, "bf16", 1e-38, 1), (2, 20, 30, "fp32", 3e-45, 1)])
def test_update_of_the_largest_and_smallest_values(L, M, N, dt, scale, steps):
    """Sums of squares far out of fp32's range, subnormals, and either side of where another scale takes over."""
    _check_ortho(L, M, N, dt, scale=scale, steps=steps, eps=0.0, seed=N)


@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("dt", DT)
def test_update_of_values_that_are_not_finite(dt, steps):
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(5, 40, 60, device="cuda", generator=g).to(types[dt])
    for i, bad in ((1, float("inf")), (2, -float("inf")), (3, float("nan"))):
        x[i, 3 * i, 7] = bad
    y = nets.orthogonalise(x, steps)
    assert torch.isfinite(y[0]).all() and torch.isfinite(y[4]).all() and torch.isnan(y[1:4]).all()
    assert torch.isnan(nets.orthogonalise(torch.zeros(1, 4, 5, device="cuda", dtype=types[dt]), steps, eps=0.0)).all()


def test_update_beside_a_large_eps():
    torch, nets, _ = _t()
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(2, 20, 30, device="cuda", generator=g) * 1e-25
    for eps in (1e-3, 1e5, 1e10):
        # a sum, a quotient and two products, 4 U; |x| is 2^-70 of eps or less; a result below 2^-126 (x of 1e-28 over 1e10) is
        # rounded to a multiple of 2^-149, off by half of that
        want = _np(x) / eps
        assert (np.abs(_np(nets.orthogonalise(x, 0, eps=eps)) - want) <= 4 * R.U * np.abs(want) + 2.0 ** -150).all()


def test_update_large():
    _check_ortho(1, 1024, 1300, "fp32", seed=1)
    _check_ortho(2, 1100, 600, "bf16", seed=2)


@pytest.mark.parametrize("L,M,N,dt,layout", [(24, 512, 640, "fp32", "flat"), (20, 700, 400, "bf16", "pad"), (24, 515, 1000, "fp32", "odd"),
                                             (24, 1000, 515, "fp16", "odd"), (20, 512, 1024, "fp32", "flat")])
def test_update_of_stacks(L, M, N, dt, layout):
    """Enough tiles for pairs of blocks, whole and ragged, either way round."""
    _check_ortho(L, M, N, dt, layout, seed=L)


@pytest.mark.parametrize("steps", [1, 2])
@pytest.mark.parametrize("L,M,N", list(zip((20, 54, 4, 27, 9, 55, 19, 52, 18, 19), *zip(*R.RANK_ONE))))
def test_update_has_all_pieces_of_its_products(L, M, N, steps):
    """Matrices of one rank with random signs, at sizes that take all kinds of tiles (one tile, narrow and wide ones, pairs of
    blocks): every value to 3e-5 of itself (1.4e-4 after two steps), a third of what a lost product of pieces would be."""
    torch, nets, _ = _t()
    g = torch.Generator(device="cuda").manual_seed(L)
    sign = lambda *s: torch.randint(0, 2, s, device="cuda", generator=g).float() * 2 - 1      # noqa: E731
    signs = sign(L, M, 1) * sign(L, 1, N)
    y = nets.orthogonalise(signs * 1e-3, steps, coef=R.RANK_ONE_COEF, eps=0.0)
    off = np.abs(_np(y * signs) * np.sqrt(M * N) - 1).max()
    assert off <= R.rank_one_bound(M, N, steps, R.RANK_ONE_COEF), off


def test_update_of_zeros_and_of_nothing():
    torch, nets, _ = _t()
    z = torch.zeros(2, 10, 20, device="cuda")
    assert not nets.orthogonalise(z).any()
    z[1, 3, 4] = float("nan")
    y = nets.orthogonalise(z)
    assert not y[0].any() and torch.isnan(y[1]).all()
    for shape in ((0, 4, 4), (2, 0, 4), (2, 4, 0)):
        assert nets.orthogonalise(torch.zeros(shape, device="cuda")).shape == shape


def test_update_in_place_and_of_infinite_values():
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(4)
    for steps in (0, 1, 5):
        for dt in DT:
            x = torch.randn(3, 40, 60, device="cuda", generator=g).to(types[dt])
            want = nets.orthogonalise(x, steps)
            assert nets.orthogonalise(x, steps, y=x) is x and torch.equal(x, want)
    x = torch.randn(2, 40, 60, device="cuda", generator=g)
    x[1, 3, 7] = float("inf")
    y = nets.orthogonalise(x)
    assert torch.isfinite(y[0]).all() and torch.isnan(y[1]).all()


def test_updates_on_two_streams_at_once():
    """Each takes the whole device and its blocks wait for one another."""
    torch, nets, _ = _t()
    g = torch.Generator(device="cuda").manual_seed(5)
    xs = [torch.randn(24, 512, 640, device="cuda", generator=g), torch.randn(3, 900, 1100, device="cuda", generator=g)]
    want = [nets.orthogonalise(x) for x in xs]
    torch.cuda.synchronize()
    low, high = torch.cuda.Stream(), torch.cuda.Stream(priority=-1)
    got = []
    for _ in range(4):
        for x, s in zip(xs, (low, high)):
            with torch.cuda.stream(s):
                got.append((nets.orthogonalise(x), torch.randn(2048, 2048, device="cuda") @ torch.randn(2048, 2048, device="cuda")))
    torch.cuda.synchronize()
    for i, (y, _) in enumerate(got):
        assert torch.equal(y, want[i % 2])


@pytest.mark.parametrize("dt,L,M,N", [("fp32", 2, 300, 200), ("bf16", 3, 150, 700), ("fp32", 24, 512, 640), ("fp16", 24, 640, 512)])
def test_update_whose_wait_gives_up(dt, L, M, N):
    """One block waits behind a product for what never comes (20 ms): the code says so, no value of y is anything but right or
    NaN, none is right where products were still to come for all blocks, and the next call is as ever.  By single blocks and by
    pairs."""
    torch, nets, types = _t()
    from paper_2512_13359_gb300.nets import NET_DTYPE, _ORTHO
    lib, t, steps = nets.lib(), types[dt], 2
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn(L, M, N, device="cuda", generator=g).to(t)
    want = nets.orthogonalise(x, steps)
    y = torch.empty_like(x)
    fields = (_ORTHO.size, NET_DTYPE[t], steps, 1e-7, 3.4445, -4.775, 2.0315, 0, L, M, N, x.data_ptr(), M * N, N, y.data_ptr(), M * N, N)
    need = lib.net_orthogonalise_workspace_bytes(_ORTHO.pack(*fields, 0, 0))
    work = torch.empty(need, device="cuda", dtype=torch.uint8)
    args = _ORTHO.pack(*fields, work.data_ptr(), need)
    code = lambda: int(work[:4].view(torch.int32).item())         # noqa: E731
    for product in range(1, 3 * steps):
        y.zero_()
        assert lib.net_orthogonalise_selftest_timeout(args, product, 20000, torch.cuda.current_stream().cuda_stream) == 0
        assert code() == -4
        gone = torch.isnan(y)
        assert gone.any() and torch.equal(y[~gone], want[~gone])
        assert gone.all() or product == 3 * steps - 1
    assert lib.net_orthogonalise(args, torch.cuda.current_stream().cuda_stream) == 0
    assert code() == 0 and torch.equal(y, want)


def test_update_of_many_small_ones():
    torch, nets, _ = _t()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(300, 12, 8, device="cuda", generator=g)
    y = nets.orthogonalise(x)
    for i in (0, 1, 150, 299):
        assert torch.equal(y[i:i + 1], nets.orthogonalise(x[i:i + 1].clone()))


# ------------------------------------------------------------ calls
def _everything(torch, nets, types, stream=None):
    """One call of each operator and its gradient; their inputs; their outputs."""
    T, N, D, S, K = 300, 2, 40, 16, 4
    g, a, opt, h0 = _scan_args(torch, types["bf16"], T, N, D, S, 1, "flat", 0.05, 11)
    w, b = torch.randn(K, D, device="cuda", generator=g), torch.randn(D, device="cuda", generator=g)
    dy = torch.randn(T, N, D, device="cuda", generator=g).to(torch.bfloat16)
    M = torch.randn(3, 70, 50, device="cuda", generator=g)
    ends = dict(done=opt["done"], done_prev=opt["done_prev"])

    def run(stream=None):
        u, new = nets.causal_conv(a["x"], w, b, act="silu", **ends, stream=stream)
        y, hT, kept = nets.select_scan(u, *(a[k] for k in ("dt", "A", "B", "C")), **opt, h0=h0, kept=True, stream=stream)
        back = nets.select_scan_backward(u, *(a[k] for k in ("dt", "A", "B", "C")), kept, dy, **opt, stream=stream)
        conv = nets.causal_conv_backward(a["x"], w, b, back[0], act="silu", **ends, stream=stream)
        return [u, new, y, hT, kept, *back, *conv, nets.orthogonalise(M, stream=stream)]
    return run


def _same(torch, p, q):
    assert len(p) == len(q) and all(torch.equal(x, y) for x, y in zip(p, q))


def test_repeated_calls_other_streams_and_graphs_give_the_same_bits():
    torch, nets, types = _t()
    run = _everything(torch, nets, types)
    want = run()
    for _ in range(3):
        _same(torch, run(), want)
    side = torch.cuda.Stream()
    got = run(stream=side)
    torch.cuda.synchronize()
    _same(torch, got, want)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = run()
        other = torch.cuda.CUDAGraph()
        with torch.cuda.graph(other, stream=side):
            held2 = run()
    for _ in range(3):
        for x in (*held, *held2):
            x.zero_()
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        _same(torch, held, want)
        _same(torch, held2, want)


def test_two_streams_at_once():
    torch, nets, types = _t()
    run = _everything(torch, nets, types)
    want = run()
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(4):
        for q in s:
            with torch.cuda.stream(q):
                got.append(run())
    torch.cuda.synchronize()
    for p in got:
        _same(torch, p, want)


def test_refusals():
    torch, nets, _ = _t()
    from paper_2512_13359_gb300.auvenv import AuvError
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)       # noqa: E731
    x, w, A, B = z(5, 3, 8), z(4, 8), z(8, 4), z(5, 3, 4)
    kept = z(1, 3, 8, 4)
    bad = [
        (-1, lambda: nets.causal_conv(x, z(4, 9))), (-1, lambda: nets.causal_conv(x, w.half())), (-6, lambda: nets.causal_conv(x, z(9, 8))),
        (-1, lambda: nets.causal_conv(x, w, act="relu")), (-1, lambda: nets.causal_conv(x, z(0, 8))),
        (-1, lambda: nets.causal_conv(x, w, None, z(2, 3, 8))), (-1, lambda: nets.causal_conv(x, w, None, z(3, 3, 8).half())),
        (-2, lambda: nets.causal_conv(x, w, None, z(3, 3, 16)[..., ::2])), (-1, lambda: nets.causal_conv(x, w, done=z(4, 3, dtype=torch.uint8))),
        (-2, lambda: nets.causal_conv(x, w, y=z(1, 3, 8).expand(5, 3, 8))), (-1, lambda: nets.causal_conv(x, w, y=x.half())),
        (-1, lambda: nets.causal_conv_backward(x, w, None, x[:4])), (-1, lambda: nets.causal_conv(x, w.cpu())),
        (-1, lambda: nets.select_scan(x, x[:4], A, B, B)), (-1, lambda: nets.select_scan(x, x, A, B, B.half())),
        (-1, lambda: nets.select_scan(x, x, A, z(5, 3, 6), z(5, 3, 6))), (-1, lambda: nets.select_scan(x, x, A, z(5, 3, 12), z(5, 3, 12))),
        (-1, lambda: nets.select_scan(x, x, A.half(), B, B)), (-6, lambda: nets.select_scan(x, x, z(8, 129), z(5, 3, 129), z(5, 3, 129))),
        (-2, lambda: nets.select_scan(x, x, z(4, 8).t(), B, B)), (-1, lambda: nets.select_scan(x, x, A, B, B, h0=z(3, 8))),
        (-1, lambda: nets.select_scan(x, x, A, B, B, kept=z(2, 3, 8, 4))), (-1, lambda: nets.select_scan(x, x, A, B, B, skip=z(7))),
        (-1, lambda: nets.select_scan_backward(x, x, A, B, B, None, x)), (-1, lambda: nets.select_scan_backward(x, x, A, B, B, z(2, 3, 8, 4), x)),
        (-1, lambda: nets.select_scan_backward(x, x, A, B, B, kept, x, dgate=x)),
        (-2, lambda: nets.select_scan_backward(x, x, A, B, B, kept, x, dB=z(1, 3, 4).expand(5, 3, 4))),
        (-1, lambda: nets.orthogonalise(x, 65)), (-1, lambda: nets.orthogonalise(x, -1)), (-1, lambda: nets.orthogonalise(x, 2.5)),
        (-1, lambda: nets.orthogonalise(x, coef=(1.0, 2.0))), (-1, lambda: nets.orthogonalise(x, coef=None)),
        (-6, lambda: nets.orthogonalise(x, coef=(9.0, 0.0, 0.0))), (-1, lambda: nets.orthogonalise(x, eps=-1.0)),
        (-1, lambda: nets.orthogonalise(x, y=x.half())), (-2, lambda: nets.orthogonalise(x, y=z(1, 3, 8).expand(5, 3, 8))),
    ]
    for i, (code, f) in enumerate(bad):
        with pytest.raises(AuvError) as e:
            f()
        assert e.value.code == code, (i, e.value)


# ------------------------------------------------------------ together
def test_a_layer_of_them_is_trained():
    """Convolution and scan as a memory of the rollout, gradients against torch's differentiation in 64 bits, and the weight
    update of its projection orthogonalised."""
    torch, nets, _ = _t()
    g = torch.Generator(device="cuda").manual_seed(21)
    rn = lambda *s: torch.randn(s, device="cuda", generator=g)    # noqa: E731
    T, N, O, D, S, K = 24, 6, 18, 16, 8, 4
    obs, W, w = rn(T, N, O), rn(4 * D + 2 * S, O) * O ** -0.5, rn(K, D) * 0.5
    b, A, skip, bias = rn(D) * 0.1, -torch.exp(rn(D, S) * 0.3), rn(D), rn(D) - 2
    done, prev = _ends(torch, T, N, 0.1, g)
    dy = rn(T, N, D)

    def halves(z):
        return z[..., :D], z[..., D:2 * D], z[..., 2 * D:3 * D], z[..., 3 * D:4 * D], z[..., 4 * D:4 * D + S], z[..., 4 * D + S:]
    z = obs @ W.t()
    x, gate, dt, _, B, C = halves(z)
    u, _ = nets.causal_conv(x, w, b, done=done, done_prev=prev, act="silu")
    y, _, kept = nets.select_scan(u, dt, A, B, C, skip=skip, dt_bias=bias, gate=gate, done=done, done_prev=prev, kept=True)
    dz = torch.zeros_like(z)
    dx, dgate, ddt, _, dB, dC = halves(dz)
    du, _, dA, _, _, dskip, dbias, _, _ = nets.select_scan_backward(u, dt, A, B, C, kept, dy, skip=skip, dt_bias=bias, gate=gate, done=done,
                                                                   done_prev=prev, ddt=ddt, dB=dB, dC=dC, dgate=dgate)
    _, dw, db, _ = nets.causal_conv_backward(x, w, b, du, done=done, done_prev=prev, act="silu", dx=dx)
    dW = dz.reshape(-1, z.shape[-1]).t() @ obs.reshape(-1, O)
    upd = nets.orthogonalise(dW[None])[0]
    leaves = [v.double().requires_grad_() for v in (W, w, b, A, skip, bias)]
    W6, w6, b6, A6, k6, s6 = leaves
    x6, gate6, dt6, _, B6, C6 = halves(obs.double() @ W6.t())
    win, h, loss = [torch.zeros(N, D, device="cuda", dtype=torch.float64)] * (K - 1), torch.zeros(N, D, S, device="cuda", dtype=torch.float64), 0.0
    silu = torch.nn.functional.silu
    for t in range(T):
        end = (prev if t == 0 else done[t - 1]).bool()[:, None]
        rows = [*(q.masked_fill(end, 0.0) for q in win), x6[t]]
        u6 = silu(sum(q * k for q, k in zip(rows, w6)) + b6)
        e = torch.nn.functional.softplus(dt6[t] + s6)
        h = torch.exp(e[..., None] * A6) * h.masked_fill(end[..., None], 0.0) + (e * u6)[..., None] * B6[t][:, None]
        y6 = ((h * C6[t][:, None]).sum(-1) + k6 * u6) * silu(gate6[t])
        loss = loss + (y6 * dy[t].double()).sum()
        win = rows[1:]
    ref = torch.autograd.grad(loss, leaves)
    for q, r in zip((dW, dw, db, dA, dskip, dbias), ref):
        # sums of T N rows, each some hundred roundings off; 3e-5 of the norm is 500 units
        assert (q.double() - r).norm() <= 3e-5 * r.norm()
    want, E = R.orthogonalise(_np(dW), 5, (3.4445, -4.775, 2.0315), 1e-7)
    assert np.linalg.norm(_np(upd) - want) <= E + R.U * np.linalg.norm(want)
