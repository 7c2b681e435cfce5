"""The network operators on a GPU against the 64-bit reference (nets_ref.py), whose bounds come with it: types, odd and
ragged sizes, lengths from none to 70,001, strides, episode ends everywhere, infinities and NaN behind them, gradients by
differences, other streams, CUDA graphs, repeated calls bit for bit, refusals."""
import numpy as np
import pytest

import nets_ref as R
from parity_util import need_gpu

pytestmark = pytest.mark.gpu

DT = ("fp32", "bf16", "fp16")


def _t():
    torch = need_gpu()
    from paper_2512_13359_gb300 import nets
    return torch, nets, {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _np(x):
    return x.detach().double().cpu().numpy()


def _rows(torch, shape, dtype, layout, gen, scale=1.0, shift=0.0):
    """A [i, j, k] tensor of normal values: contiguous, with rows that start off any vector's boundary ("odd") or on one
    ("pad"), one half of a wider array ("half"), or with the first two axes swapped in memory ("swap")."""
    i, j, k = shape
    full = {"odd": (i, j, k + 3), "pad": (i, j, k + 16), "half": (i, j, 2 * k), "swap": (j, i, k)}.get(layout, shape)
    x = (torch.randn(full, device="cuda", generator=gen) * scale + shift).to(dtype)
    if layout == "swap":
        return x.transpose(0, 1)
    return x[..., 1:1 + k] if layout == "odd" else x[..., k:] if layout == "half" else x[..., :k]


def _within(got, ref, E, dtype="fp32"):
    bound = R.stored(ref, E, dtype)
    d = np.abs(_np(got) - ref)
    assert np.isfinite(d).all()
    worst = (d / bound).max() if d.size else 0.0
    assert worst <= 1.0, f"{worst:.2f} of the bound"


def _scan_inputs(torch, T, N, D, dtype, layout, ends, seed, state=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    f = _rows(torch, (T, N, D), dtype, layout, g, 1.5, 1.5)
    v = _rows(torch, (T, N, D), dtype, layout, g)
    h0 = torch.randn((N, D), device="cuda", generator=g) if state else None
    done = prev = None
    if ends is not None:
        done = (torch.rand((T, N), device="cuda", generator=g) < ends).to(torch.uint8)
        prev = (torch.rand((N,), device="cuda", generator=g) < max(ends, 0.3)).to(torch.uint8)
    return g, f, v, h0, done, prev


def _check_scan(T, N, D, dt, layout="flat", ends=0.1, seed=0, state=True):
    torch, nets, types = _t()
    g, f, v, h0, done, prev = _scan_inputs(torch, T, N, D, types[dt], layout, ends, seed, state)
    nn = lambda x: None if x is None else _np(x)                 # noqa: E731
    y = _rows(torch, (T, N, D), types[dt], layout, g)
    y, hT = nets.gate_scan(f, v, h0, done=done, done_prev=prev, y=y)
    ry, rh, Ey, Eh = R.gate_scan(_np(f), _np(v), nn(h0), nn(done), nn(prev))
    _within(y, ry, Ey, dt)
    _within(hT, rh, Eh)
    dy = _rows(torch, (T, N, D), types[dt], layout, g, 0.5)
    dhT = torch.randn((N, D), device="cuda", generator=g) if state else None
    df, dv = (_rows(torch, (T, N, D), types[dt], layout, g) for _ in range(2))
    df, dv, dh0 = nets.gate_scan_backward(f, v, y, dy, h0, done=done, done_prev=prev, dhT=dhT, df=df, dv=dv)
    r = R.gate_scan_backward(_np(f), _np(v), _np(y), _np(dy), nn(h0), nn(done), nn(prev), nn(dhT))
    _within(df, r[0], r[3], dt)
    _within(dv, r[1], r[4], dt)
    _within(dh0, r[2], r[5])


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,N,D", [(1, 1, 256), (1, 700, 40), (2, 3, 5), (7, 33, 12), (8, 5, 64), (33, 4, 100),
                                   (129, 2, 250), (300, 9, 17), (1000, 3, 64), (257, 1, 1), (9, 3000, 24)])
def test_recurrence(T, N, D, dt):
    _check_scan(T, N, D, dt, seed=T)


@pytest.mark.parametrize("layout", ["odd", "pad", "half", "swap"])
@pytest.mark.parametrize("T,N,D,dt", [(20, 6, 24, "bf16"), (20, 6, 24, "fp32"), (3, 5000, 16, "bf16"), (700, 3, 16, "bf16"),
                                      (700, 3, 16, "fp32"), (700, 2, 33, "fp16")])
def test_recurrence_strides(T, N, D, dt, layout):
    _check_scan(T, N, D, dt, layout, seed=5)


@pytest.mark.parametrize("ends", [None, 0.0, 0.6, 1.0])
@pytest.mark.parametrize("T,N,D", [(40, 50, 32), (1500, 2, 24), (1, 4, 8)])
def test_recurrence_ends(T, N, D, ends):
    _check_scan(T, N, D, "fp32", ends=ends, seed=6, state=ends != 0.6)


@pytest.mark.parametrize("T,N,D,dt", [(70001, 1, 3, "fp32"), (70001, 1, 4, "bf16"), (20000, 2, 12, "fp16"),
                                      (5000, 1, 96, "bf16")])
def test_recurrence_long(T, N, D, dt):
    _check_scan(T, N, D, dt, ends=0.0005, seed=7)


@pytest.mark.parametrize("layout,T,N,D,dt", [("half", 30011, 1, 40, "bf16"), ("odd", 30011, 2, 33, "fp16"), ("swap", 20003, 2, 48, "fp32"),
                                             ("pad", 25000, 3, 17, "fp32"), ("flat", 20003, 1, 250, "bf16"), ("flat", 16385, 4, 63, "fp16")])
def test_recurrence_long_strides(layout, T, N, D, dt):
    _check_scan(T, N, D, dt, layout, ends=0.0005, seed=12)


@pytest.mark.parametrize("N,D,dt", [(40000, 256, "bf16"), (33333, 33, "fp16"), (70000, 64, "fp32")])
def test_recurrence_wide(N, D, dt):
    _check_scan(3, N, D, dt, seed=8)


def test_recurrence_without_steps_or_envs():
    torch, nets, types = _t()
    h0 = torch.randn(4, 8, device="cuda")
    z = torch.empty(0, 4, 8, device="cuda")
    y, hT = nets.gate_scan(z, z, h0)
    assert y.numel() == 0 and torch.equal(hT, h0)
    assert torch.equal(nets.gate_scan(z, z)[1], torch.zeros_like(h0))
    assert torch.equal(nets.gate_scan_backward(z, z, z, z, h0, dhT=2 * h0)[2], 2 * h0)
    z = torch.empty(5, 0, 8, device="cuda")
    assert nets.gate_scan(z, z)[0].shape == (5, 0, 8)


@pytest.mark.parametrize("T", [12, 900, 60000])
@pytest.mark.parametrize("dt", DT)
def test_nothing_of_an_ended_episode_passes(T, dt):
    """Infinities and NaN in an ended episode's inputs and state: finite after its end, and the gradients before an end
    are those of its own steps alone."""
    torch, nets, types = _t()
    g, f, v, h0, done, prev = _scan_inputs(torch, T, 3, 40, types[dt], "flat", 0.0, 9)
    cut = T // 2
    done[cut - 1, :2] = 1
    prev[:] = torch.tensor([1, 0, 1], device="cuda")
    want = nets.gate_scan(f, v, h0, done=done, done_prev=prev)
    bad = [x.clone() for x in (f, v, h0)]
    bad[2][0] = float("nan")                      # ended before step 0
    bad[1][cut - 3, 0], bad[1][cut - 2, 1], bad[0][cut - 1, 1] = float("inf"), float("nan"), float("nan")
    y, hT = nets.gate_scan(*bad, done=done, done_prev=prev)
    assert torch.equal(hT, want[1]) and torch.equal(y[cut:], want[0][cut:]) and torch.equal(y[:, 2], want[0][:, 2])
    assert torch.equal(y[:cut - 3, 0], want[0][:cut - 3, 0]) and not torch.isfinite(y[cut - 1, :2]).any()
    dy = torch.randn((T, 3, 40), device="cuda", generator=g).to(types[dt])
    ref = nets.gate_scan_backward(f, v, want[0], dy, h0, done=done, done_prev=prev)
    dyb, yb = dy.clone(), want[0].clone()
    dyb[cut + 1, :2] = float("nan")               # the gradient after the end
    yb[cut - 1, :2] = float("inf")                # the state that was cut off
    got = nets.gate_scan_backward(f, v, yb, dyb, bad[2], done=done, done_prev=prev)
    for a, b in zip(got[:2], ref[:2]):
        assert torch.equal(a[:cut], b[:cut]) and torch.equal(a[:, 2], b[:, 2]) and torch.equal(a[cut + 2:], b[cut + 2:])
    assert torch.equal(got[2], ref[2]) and (got[2][0] == 0).all()


@pytest.mark.parametrize("T", [5, 600])
def test_gates_wide_open_and_shut(T):
    """f = +-inf and the type's lowest and largest values: the gate is 1 or 0, nothing is NaN."""
    torch, nets, types = _t()
    for dt in DT:
        f = torch.empty((T, 1, 8), device="cuda", dtype=types[dt])
        lim = torch.finfo(types[dt])
        f[..., 0::4], f[..., 1::4], f[..., 2::4], f[..., 3::4] = float("inf"), float("-inf"), lim.min, lim.max
        v = torch.randn((T, 1, 8), device="cuda").to(types[dt])
        h0 = torch.randn((1, 8), device="cuda")
        y, hT = nets.gate_scan(f, v, h0)
        keep = h0.to(types[dt]).expand(T, 8)
        for k in (0, 3):
            assert torch.equal(y[:, 0, k::4], keep[:, k::4])
        for k in (1, 2):
            assert torch.equal(y[:, 0, k::4], v[:, 0, k::4])
        df, dv, dh0 = nets.gate_scan_backward(f, v, y, torch.ones_like(v), h0)
        assert (df == 0).all() and (dv[..., 1::4] == 1).all() and (dv[..., 0::4] == 0).all() and (dh0[:, 0::4] == T).all()


def test_recurrence_gradient_by_differences():
    torch, nets, types = _t()
    for T, N, D in ((9, 4, 8), (400, 1, 12)):
        g, f, v, h0, done, prev = _scan_inputs(torch, T, N, D, torch.float32, "flat", 0.02, 10)
        dy, dhT = torch.randn((T, N, D), device="cuda", generator=g), torch.randn((N, D), device="cuda", generator=g)
        y, _ = nets.gate_scan(f, v, h0, done=done, done_prev=prev)
        grads = nets.gate_scan_backward(f, v, y, dy, h0, done=done, done_prev=prev, dhT=dhT)
        args = [_np(q) for q in (f, v, h0)]

        def loss(f, v, h0):
            y, hT, _, _ = R.gate_scan(f, v, h0, _np(done), _np(prev))
            return (y * _np(dy)).sum() + (hT * _np(dhT)).sum()
        rng = np.random.default_rng(1)
        for k in range(3):
            d, e = rng.normal(size=args[k].shape), 1e-5
            hi, lo = (loss(*[q + s * e * d if i == k else q for i, q in enumerate(args)]) for s in (1, -1))
            terms = _np(grads[k]) * d
            # central differences: 1e-10 of the third derivative; the kernel's fp32: some 1e-6 of each term
            assert abs((hi - lo) / (2 * e) - terms.sum()) <= 1e-5 * np.abs(terms).sum() + 1e-8


def test_state_in_place_and_steps_equal_the_sequence():
    """A rollout's steps, each with T = 1, the state updated in place and the flags of the step before, give the
    sequence's outputs."""
    torch, nets, types = _t()
    g, f, v, h0, done, prev = _scan_inputs(torch, 20, 37, 24, torch.float32, "half", 0.2, 11)
    y, hT = nets.gate_scan(f, v, h0, done=done, done_prev=prev)
    h = h0.clone()
    for t in range(20):
        yt, out = nets.gate_scan(f[t:t + 1], v[t:t + 1], h, done_prev=prev if t == 0 else done[t - 1], hT=h)
        assert out is h
        assert torch.equal(yt[0], y[t])
    assert torch.equal(h, hT)
    b = nets.gate_scan(f, v, h0, done=done.bool(), done_prev=prev.bool())
    assert torch.equal(b[0], y) and torch.equal(b[1], hT)


def test_offsets_past_32_bits():
    """Steps 2^31 + 24 elements apart."""
    torch, nets, types = _t()
    gap = (1 << 31) + 24
    big = torch.empty(2 * gap + 4 * 16, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((3, 4, 16), (gap, 16, 1))
    src = torch.randn((3, 4, 16), device="cuda").to(torch.bfloat16)
    x.copy_(src)
    v = torch.randn((3, 4, 16), device="cuda").to(torch.bfloat16)
    a, b = nets.gate_scan(x, v), nets.gate_scan(src, v)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    a, b = nets.group_norm(x, 4), nets.group_norm(src, 4)
    assert torch.equal(a[0], b[0])
    assert torch.equal(nets.dropout(x, 0.3, 1, 2), nets.dropout(src, 0.3, 1, 2))
    nets.gate_scan(src, v, y=x)
    assert torch.equal(x, nets.gate_scan(src, v)[0])


# ------------------------------------------------------------ group norm
def _check_norm(B, S, C, G, dt, act, layout="flat", seed=0, affine=True, shift=0.3):
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = _rows(torch, (B, S, C), types[dt], layout, g, 1.3, shift)
    dy = _rows(torch, (B, S, C), types[dt], layout, g, 0.5)
    gamma = torch.randn(C, device="cuda", generator=g) * 0.3 + 1 if affine else None
    beta = torch.randn(C, device="cuda", generator=g) * 0.3 if affine else None
    ng, nb = (_np(gamma), _np(beta)) if affine else (np.ones(C), np.zeros(C))
    y = _rows(torch, (B, S, C), types[dt], layout, g)
    y, mean, rstd = nets.group_norm(x, G, gamma, beta, eps=1e-5, act=act, y=y)
    r = R.group_norm(_np(x), G, ng, nb, 1e-5, act)
    _within(mean, r[1], r[4])
    _within(rstd, r[2], r[5])
    _within(y, r[0], r[3], dt)
    dx = _rows(torch, (B, S, C), types[dt], layout, g)
    dx, dgamma, dbeta = nets.group_norm_backward(x, G, gamma, beta, mean, rstd, dy, act=act, dx=dx)
    r = R.group_norm_backward(_np(x), G, ng, nb, _np(mean), _np(rstd), _np(dy), act)
    _within(dx, r[0], r[3], dt)
    _within(dgamma, r[1], r[4])
    _within(dbeta, r[2], r[5])


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("B,S,C,G,act", [
    (1, 1, 256, 1, "relu"), (256, 1, 90, 9, "tanh"), (1000, 1, 256, 1, "silu"), (77, 1, 64, 8, "none"),
    (5, 3, 24, 3, "silu"), (3, 100, 32, 4, "tanh"), (2, 1000, 16, 2, "relu"), (4, 37, 250, 25, "silu"),
    (1, 9, 7, 7, "none"), (130, 1, 1024, 1, "tanh"), (3, 2, 1, 1, "none"), (2, 3000, 3, 1, "silu"),
    (1, 1, 5000, 1, "silu"), (2, 700, 96, 1, "relu"), (6, 129, 128, 32, "silu"), (9, 1, 40, 20, "none")])
def test_norm(B, S, C, G, act, dt):
    _check_norm(B, S, C, G, dt, act, seed=B + C)


@pytest.mark.parametrize("layout", ["odd", "pad", "half", "swap"])
@pytest.mark.parametrize("B,S,C,G,dt", [(33, 1, 64, 2, "bf16"), (33, 1, 64, 2, "fp32"), (6, 50, 48, 6, "bf16"),
                                        (2, 900, 40, 5, "fp16"), (3, 400, 64, 1, "fp32")])
def test_norm_strides(B, S, C, G, dt, layout):
    _check_norm(B, S, C, G, dt, "silu", layout, seed=3)


@pytest.mark.parametrize("B,S,C,G,dt", [(2, 20000, 64, 8, "bf16"), (1, 70001, 33, 3, "fp32"), (1, 9000, 512, 2, "fp16"),
                                        (40, 600, 256, 32, "bf16"), (70000, 1, 24, 1, "bf16"), (20000, 2, 40, 5, "fp16")])
def test_norm_large(B, S, C, G, dt):
    _check_norm(B, S, C, G, dt, "silu", seed=4)


def test_norm_without_weights_or_values():
    torch, nets, types = _t()
    _check_norm(8, 5, 32, 4, "fp32", "silu", affine=False)
    z = torch.empty(0, 3, 8, device="cuda")
    y, mean, rstd = nets.group_norm(z, 2)
    assert y.shape == z.shape and mean.shape == (0, 2)
    dx, dg, db = nets.group_norm_backward(z, 2, None, None, mean, rstd, z)
    assert (dg == 0).all() and (db == 0).all() and dg.shape == (8,)
    z = torch.empty(3, 0, 8, device="cuda")
    y, mean, rstd = nets.group_norm(z, 2, eps=0.25)
    assert (mean == 0).all() and (rstd == 2).all()
    assert (nets.group_norm_backward(z, 2, None, None, mean, rstd, z)[1] == 0).all()


@pytest.mark.parametrize("B,S,C,G", [(16, 1, 256, 1), (3, 2000, 32, 4), (2, 20, 32, 4), (1, 40000, 64, 2)])
def test_norm_of_values_far_from_zero(B, S, C, G):
    """A mean a thousand deviations off: the variance is that of the deviations, not a difference of squares (whose
    rounding, 2^-24 of 10^6, would be 6 % of it)."""
    _check_norm(B, S, C, G, "fp32", "none", shift=1300.0)


def test_norm_constant_group_and_nonfinite_neighbours():
    torch, nets, types = _t()
    for S in (1, 300, 5000):
        x = torch.randn((4, S, 32), device="cuda")
        x[1, :, :8] = 3.0
        want = nets.group_norm(x, 4, eps=1e-5)
        assert (want[0][1, :, :8] == 0).all()
        x[2, S // 2, 9] = float("nan")                  # one group of one instance
        x[3, 0, 31] = float("inf")
        y, mean, rstd = nets.group_norm(x, 4, eps=1e-5)
        clean = torch.ones((4, S, 32), dtype=torch.bool, device="cuda")
        clean[2, :, 8:16] = clean[3, :, 24:] = False
        assert torch.equal(y[clean], want[0][clean]) and torch.isnan(y[2, :, 8:16]).all()


@pytest.mark.parametrize("act", ["none", "silu", "tanh"])
def test_norm_gradient_by_differences(act):
    torch, nets, types = _t()
    for B, S, C, G in ((5, 1, 24, 3), (2, 40, 16, 2), (1, 900, 8, 1)):
        x = torch.randn((B, S, C), device="cuda")
        gamma, beta = torch.randn(C, device="cuda") * 0.3 + 1, torch.randn(C, device="cuda") * 0.3
        dy = torch.randn((B, S, C), device="cuda")
        _, mean, rstd = nets.group_norm(x, G, gamma, beta, act=act)
        grads = nets.group_norm_backward(x, G, gamma, beta, mean, rstd, dy, act=act)
        args = [_np(q) for q in (x, gamma, beta)]
        loss = lambda x, g, b: (R.group_norm(x, G, g, b, 1e-5, act)[0] * _np(dy)).sum()  # noqa: E731
        rng = np.random.default_rng(1)
        for k in range(3):
            d, e = rng.normal(size=args[k].shape), 1e-5
            hi, lo = (loss(*[q + s * e * d if i == k else q for i, q in enumerate(args)]) for s in (1, -1))
            terms = _np(grads[k]) * d
            assert abs((hi - lo) / (2 * e) - terms.sum()) <= 1e-5 * np.abs(terms).sum() + 1e-8


# ------------------------------------------------------------ dropout
@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,N,D,p,shared,residual,layout", [
    (1, 1, 1, 0.5, False, False, "flat"), (1, 256, 256, 0.01, False, True, "flat"), (5, 7, 33, 0.25, False, True, "flat"),
    (9, 13, 17, 0.3, True, False, "flat"), (16, 12, 64, 0.1, True, True, "half"), (3, 50, 40, 0.9, False, False, "odd"),
    (7, 20, 257, 0.25, True, True, "odd"), (11, 6, 24, 0.5, False, True, "swap"), (11, 6, 24, 0.5, True, False, "swap"),
    (2, 3, 1000, 0.0, False, True, "pad"), (2, 3, 100, 1.0, True, True, "pad"), (700, 9, 8, 0.2, True, False, "flat"),
    (1, 100001, 3, 0.2, False, False, "flat"), (3, 5, 4, 0.4, False, False, "half")])
def test_dropout(T, N, D, p, shared, residual, layout, dt):
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(T + D)
    x = _rows(torch, (T, N, D), types[dt], layout, g)
    x[x == 0] = 1.0
    r = _rows(torch, (T, N, D), types[dt], layout, g) if residual else None
    seed, draw = 0xFEDCBA9876543210, 0x123456789
    y = _rows(torch, (T, N, D), types[dt], layout, g)
    nets.dropout(x, p, seed, draw, residual=r, shared=shared, y=y)
    n = N * D if shared else T * N * D
    keep = R.dropout_keep(n, p, seed, draw).reshape(1 if shared else T, N, D)
    ref = _np(x) * keep
    E = 2 * R.U * np.abs(ref)
    if residual:
        ref = ref + _np(r)
        E += 2 * R.U * np.abs(ref)
    else:
        assert np.array_equal(_np(y) != 0, np.broadcast_to(keep != 0, (T, N, D)))
    _within(y, ref, E, dt)
    in_place = x.clone()
    nets.dropout(in_place, p, seed, draw, residual=r, shared=shared, y=in_place)
    assert torch.equal(in_place, y)


def test_dropout_draws_differ_and_pass_nothing_of_the_dropped():
    torch, nets, types = _t()
    x = torch.ones((1, 64, 256), device="cuda")
    a, b = nets.dropout(x, 0.5, 1, 2), nets.dropout(x, 0.5, 1, 3)
    c = nets.dropout(x, 0.5, 1 + (1 << 32), 2)
    for q in (b, c):
        assert 0.4 < (a != q).float().mean() < 0.6
    bad = torch.where(a == 0, float("nan"), x)
    assert torch.equal(nets.dropout(bad, 0.5, 1, 2), a)
    assert (nets.dropout(bad, 1.0, 1, 2, residual=x) == 1).all()


def test_dropout_index_past_32_bits():
    """The mask of the elements past 2^32 is that of their own index: a 2^32 + 4096 element call's last rows."""
    torch, nets, types = _t()
    rows, D = (1 << 20) + 1, 4096
    x = torch.ones((1, rows, D), dtype=torch.bfloat16, device="cuda")
    nets.dropout(x, 0.5, 7, 9, y=x)
    q = np.arange(D // 8, dtype=np.uint64) + np.uint64((rows - 1) * D // 8)
    w = R.philox(q & np.uint64(0xFFFFFFFF), q >> np.uint64(32), 9, 0, 7, 0)
    bits = np.stack([w & 0xFFFF, w >> 16], axis=-1).reshape(-1)
    assert np.array_equal(_np(x[0, -1]), np.where(bits < 32768, 0.0, 2.0))


# ------------------------------------------------------------ calls
def _calls(torch, nets, B):
    """Every operator once on the buffers B."""
    y, hT = nets.gate_scan(B["f"], B["v"], B["h0"], done=B["done"], y=B["y"], hT=B["hT"], stream=B.get("stream"))
    nets.dropout(y, 0.2, 3, 4, residual=B["v"], y=B["z"], stream=B.get("stream"))
    nets.group_norm(B["z"], 4, B["w"], None, act="silu", y=B["o"], mean=B["mean"], rstd=B["rstd"], stream=B.get("stream"))
    nets.group_norm_backward(B["z"], 4, B["w"], None, B["mean"], B["rstd"], B["dy"], act="silu", dx=B["dz"],
                             dgamma=B["dg"], dbeta=B["db"], stream=B.get("stream"))
    nets.dropout(B["dz"], 0.2, 3, 4, y=B["dz"], stream=B.get("stream"))
    nets.gate_scan_backward(B["f"], B["v"], y, B["dz"], B["h0"], done=B["done"], df=B["df"], dv=B["dv"], dh0=B["dh0"],
                            stream=B.get("stream"))


OUT = ("y", "hT", "z", "o", "mean", "rstd", "dz", "dg", "db", "df", "dv", "dh0")


def _buffers(torch, T, N, D, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B = {k: torch.randn((T, N, D), device="cuda", generator=g).to(dtype) for k in ("f", "v", "dy")}
    B |= {k: torch.zeros((T, N, D), device="cuda", dtype=dtype) for k in ("y", "z", "o", "dz", "df", "dv")}
    B |= {k: torch.zeros((N, D), device="cuda") for k in ("hT", "dh0")}
    B["h0"] = torch.randn((N, D), device="cuda", generator=g)
    B["done"] = (torch.rand((T, N), device="cuda", generator=g) < 0.05).to(torch.uint8)
    B |= {k: torch.zeros(D, device="cuda") for k in ("dg", "db")}
    B["w"] = torch.randn(D, device="cuda", generator=g)
    B |= {k: torch.zeros((T, 4), device="cuda") for k in ("mean", "rstd")}
    return B


@pytest.mark.parametrize("T,N,D", [(16, 64, 32), (2000, 2, 32), (3, 9000, 64), (2, 30000, 20), (40000, 1, 64)])
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_repeated_calls_other_streams_and_graphs_agree(T, N, D, dt):
    torch, nets, types = _t()
    B = _buffers(torch, T, N, D, types[dt])
    _calls(torch, nets, B)
    want = {k: B[k].clone() for k in OUT}

    def same(what):
        torch.cuda.synchronize()
        for k in OUT:
            assert torch.equal(B[k], want[k]), (what, k)
            B[k].zero_()
        torch.cuda.synchronize()
    same("first")
    _calls(torch, nets, B)
    same("again")
    s = torch.cuda.Stream()
    B["stream"] = s
    _calls(torch, nets, B)
    s.synchronize()
    same("on another stream")
    del B["stream"]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _calls(torch, nets, B)
    for _ in range(2):
        graph.replay()
        same("replayed")


def test_outputs_allocated_for_another_stream():
    torch, nets, types = _t()
    f, v = (torch.randn((50, 40, 64), device="cuda") for _ in range(2))
    want = nets.gate_scan(f, v)[0]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [nets.gate_scan(f, v, stream=s)[0] for _ in range(8)]
    s.synchronize()
    for q in got:
        assert torch.equal(q, want)


def test_refusals():
    torch, nets, types = _t()
    from paper_2512_13359_gb300.auvenv import AUV_ERR_INVALID, AUV_ERR_SIZE, AuvError
    x = torch.randn((4, 6, 8), device="cuda")
    h = torch.zeros((6, 8), device="cuda")
    stats = torch.zeros((4, 2), device="cuda")
    cases = [
        (AUV_ERR_INVALID, lambda: nets.gate_scan(x, x[:3])),
        (AUV_ERR_INVALID, lambda: nets.gate_scan(x, x.bfloat16())),
        (AUV_ERR_SIZE, lambda: nets.gate_scan(x.transpose(1, 2), x.transpose(1, 2))),
        (AUV_ERR_INVALID, lambda: nets.gate_scan(x, x, h.half())),
        (AUV_ERR_SIZE, lambda: nets.gate_scan(x, x, h.t().contiguous().t())),
        (AUV_ERR_INVALID, lambda: nets.gate_scan(x, x, done=torch.zeros((4, 6), device="cuda"))),
        (AUV_ERR_INVALID, lambda: nets.gate_scan(x, x, done=torch.zeros((4, 6), dtype=torch.uint8))),
        (AUV_ERR_SIZE, lambda: nets.gate_scan(x, x, y=torch.empty((1, 6, 8), device="cuda").expand(4, 6, 8))),
        (AUV_ERR_SIZE, lambda: nets.gate_scan(x, x, y=torch.empty(64, device="cuda").as_strided((4, 6, 8), (8, 4, 1)))),
        (AUV_ERR_INVALID, lambda: nets.gate_scan_backward(x, x, x, x[..., :4])),
        (AUV_ERR_INVALID, lambda: nets.group_norm(x, 3)),
        (AUV_ERR_INVALID, lambda: nets.group_norm(x, 0)),
        (AUV_ERR_INVALID, lambda: nets.group_norm(x, 2, act="gelu")),
        (AUV_ERR_INVALID, lambda: nets.group_norm(x, 2, eps=-1.0)),
        (AUV_ERR_INVALID, lambda: nets.group_norm(x, 2, torch.ones(4, device="cuda"))),
        (AUV_ERR_INVALID, lambda: nets.group_norm_backward(x, 2, None, None, stats, stats[:, :1], x)),
        (AUV_ERR_INVALID, lambda: nets.dropout(x, -0.1, 0, 0)),
        (AUV_ERR_INVALID, lambda: nets.dropout(x, 0.1, 0, 0, residual=x[:2])),
    ]
    for code, bad in cases:
        with pytest.raises(AuvError) as e:
            bad()
        assert e.value.code == code, str(e.value)
    L, z, r = nets.lib(), nets._NO_ROWS, (x.data_ptr(), 48, 8)
    out, other = torch.empty_like(x), torch.empty_like(stats)
    norm = (nets._NORM.size, 0, 0, 1e-5, 4, 6, 8, 2, *r, out.data_ptr(), 48, 8, *z, *z, 0, 0, stats.data_ptr(),
            other.data_ptr(), 0, 0)
    assert L.net_group_norm(nets._NORM.pack(*norm, 0, 0), 0) == 0
    host = torch.zeros(4, 6, 8)
    bad = (nets._NORM.size, 0, 0, 1e-5, 4, 6, 8, 2, host.data_ptr(), 48, 8, *norm[11:])
    assert L.net_group_norm(nets._NORM.pack(*bad, 0, 0), 0) == AUV_ERR_SIZE and b"device memory" in L.net_last_error()
    long = torch.zeros((40000, 1, 64), device="cuda")
    q = (long.data_ptr(), 64, 64)
    scan = (nets._SCAN.size, 0, 40000, 1, 64, *q, *q, *q, *z, *z, *z, *(6 * (0,)))
    need = L.net_gate_scan_workspace_bytes(nets._SCAN.pack(*scan, 0, 0), 0)
    assert need > 0
    assert L.net_gate_scan(nets._SCAN.pack(*scan, 0, need), 0) == AUV_ERR_INVALID and b"workspace" in L.net_last_error()
    assert L.net_gate_scan(nets._SCAN.pack(*scan, long.data_ptr(), need - 1), 0) == AUV_ERR_SIZE
    torch.cuda.synchronize()                     # nothing was launched that could have gone wrong
    y, hT = nets.gate_scan(x, x[:1].expand(4, 6, 8))                 # repeated inputs are fine
    assert torch.equal(y, nets.gate_scan(x, x[:1].expand(4, 6, 8).contiguous())[0])
