"""The network operators on a GPU where their plans change and where fp32 ends, against the 64-bit reference
(nets_ref.py)."""
import numpy as np
import pytest

import nets_ref as R
from test_gpu_nets import DT, _check_norm, _check_scan, _np, _t, _within

pytestmark = pytest.mark.gpu


def _shapes_of_every_way():
    return [(300, 1, 64, 2, 0), (20, 30, 40, 5, 0), (40, 550, 80, 10, 0), (3, 600, 64, 1, 1), (1, 9000, 33, 3, 0)]


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("B,S,C,G,off", _shapes_of_every_way())
def test_tanh_keeps_its_precision_near_zero(B, S, C, G, off, dt):
    """|u| from 1e-9 to 1: a relative error of fp32's size, so a 16-bit result is the rounded one or its neighbour."""
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(35)
    x = torch.randn((B, S, C + off), device="cuda", generator=g).to(types[dt])[..., off:]
    gamma = 10.0 ** (torch.rand(C, device="cuda", generator=g) * 9 - 9)
    y, mean, rstd = nets.group_norm(x, G, gamma, act="tanh")
    xg = _np(x).reshape(B, S, G, C // G)
    dev = xg - _np(mean)[:, None, :, None]
    xh = (dev * _np(rstd)[:, None, :, None]).reshape(B, S, C)     # from the call's own statistics
    u = _np(gamma) * xh
    # a difference (u of its terms), two products; tanh's slope is at most 1, its own error 16 u of its value
    terms = ((np.abs(xg) + np.abs(_np(mean))[:, None, :, None]) * _np(rstd)[:, None, :, None]).reshape(B, S, C)
    E = _np(gamma) * R.U * (2 * terms + 4 * np.abs(xh)) + 16 * R.U * np.abs(np.tanh(u))
    _within(y, np.tanh(u), E, dt)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("shift", [0.0, 4.0, -9.0, 20.0])
@pytest.mark.parametrize("B,S,C,G,off", _shapes_of_every_way())
def test_tanh_slope_keeps_its_precision(B, S, C, G, off, shift, dt):
    """1 - tanh^2 where tanh saturates: 1.7e-17 at u = 20, of which a difference from 1 has no digit."""
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(36)
    x, dy = (torch.randn((B, S, C + off), device="cuda", generator=g).to(types[dt])[..., off:] for _ in range(2))
    gamma = torch.rand(C, device="cuda", generator=g) * 0.3 + 0.1
    beta = torch.randn(C, device="cuda", generator=g) * 0.1 + shift
    _, mean, rstd = nets.group_norm(x, G, gamma, beta)
    got = nets.group_norm_backward(x, G, gamma, beta, mean, rstd, dy, act="tanh")
    U, ng, nb = R.U, _np(gamma), _np(beta)
    xg, m, r = _np(x).reshape(B, S, G, C // G), _np(mean)[:, None, :, None], _np(rstd)[:, None, :, None]
    xh = ((xg - m) * r).reshape(B, S, C)
    Exh = (2 * U * (np.abs(xg) + np.abs(m)) * r).reshape(B, S, C) + U * np.abs(xh)
    u = ng * xh + nb
    Eu = ng * Exh + 3 * U * (np.abs(ng * xh) + np.abs(nb))
    slope = 1 / np.cosh(u) ** 2
    dz = _np(dy) * slope
    # relative: of the slope by u, -2 tanh(u); its own, an exponential of 2 |u| (rounded: 2 |u|) and some ten roundings
    Edz = np.abs(dz) * (2 * Eu + U * (4 * np.abs(u) + 32))
    w, Ew = ng * dz, ng * (Edz + U * np.abs(dz))
    split = lambda q: q.reshape(B, S, G, C // G)                   # noqa: E731
    avg = lambda q: q.mean(axis=(1, 3), keepdims=True)             # noqa: E731
    w, Ew, xs, Exs = split(w), split(Ew), split(xh), split(Exh)
    k, kb = R._sum_error(S * (C // G)), R._sum_error(B * S)
    m1, m2 = avg(w), avg(w * xs)
    E1, E2 = avg(Ew) + k * avg(np.abs(w)), avg(Ew * np.abs(xs) + np.abs(w) * Exs) + k * avg(np.abs(w * xs))
    dx = r * (w - m1 - xs * m2)
    Edx = r * (Ew + E1 + np.abs(xs) * E2 + np.abs(m2) * Exs + 4 * U * (np.abs(w) + np.abs(m1) + np.abs(xs * m2)))
    _within(got[0], dx.reshape(B, S, C), Edx.reshape(B, S, C), dt)
    _within(got[1], (dz * xh).sum(axis=(0, 1)),
            (Edz * np.abs(xh) + np.abs(dz) * Exh).sum(axis=(0, 1)) + kb * np.abs(dz * xh).sum(axis=(0, 1)))
    _within(got[2], dz.sum(axis=(0, 1)), Edz.sum(axis=(0, 1)) + kb * np.abs(dz).sum(axis=(0, 1)))


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("B,S,C,G,off", [(16, 1, 256, 1, 0), (3, 700, 24, 3, 1), (9, 40, 250, 1, 0), (200, 550, 80, 10, 0),
                                         (3, 5000, 64, 2, 0), (3, 5000, 64, 2, 1), (1, 40000, 33, 3, 0)])
def test_norm_of_values_whose_variance_overflows(B, S, C, G, off, dt):
    """The sum of squares passes fp32: rstd is 0 and every value its beta, whichever way is taken."""
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(34)
    x = (torch.randn((B, S, C + off), device="cuda", generator=g) * 1e25).to(types[dt])[..., off:]
    beta = torch.randn(C, device="cuda", generator=g)
    dy = torch.randn((B, S, C), device="cuda", generator=g).to(types[dt])
    y, mean, rstd = nets.group_norm(x, G, None, beta, act="tanh")
    assert (rstd == 0).all() and torch.isfinite(mean).all()
    assert torch.equal(y, y[:1, :1].expand_as(y))
    _within(y[0, 0], np.tanh(_np(beta)), 16 * R.U * np.abs(np.tanh(_np(beta))), dt)
    dx, dgamma, dbeta = nets.group_norm_backward(x, G, None, beta, mean, rstd, dy, act="tanh")
    assert (dx == 0).all() and (dgamma == 0).all() and torch.isfinite(dbeta).all()


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("T,N,D", [(12, 3, 40), (900, 3, 40), (600, 2, 3001), (5000, 2, 96), (60000, 2, 40)])
def test_an_infinite_state_stays_infinite(T, N, D, dt):
    """No end, no gate that is 0: what is infinite once is infinite from then on, however far."""
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(24)
    f = (torch.randn((T, N, D), device="cuda", generator=g) * 0.5 + 0.5).to(types[dt])
    v, dy = (torch.randn((T, N, D), device="cuda", generator=g).to(types[dt]) for _ in range(2))
    h0 = torch.randn((N, D), device="cuda", generator=g)
    want = nets.gate_scan(f, v, h0)
    v[3, 0, ::2] = float("inf")
    h0[1, 1] = float("-inf")
    y, hT = nets.gate_scan(f, v, h0)
    assert (y[3:, 0, ::2] == float("inf")).all() and (hT[0, ::2] == float("inf")).all()
    assert (y[:, 1, 1] == float("-inf")).all() and hT[1, 1] == float("-inf")
    assert torch.equal(y[:, 0, 1::2], want[0][:, 0, 1::2]) and torch.equal(y[:, 1, 2:], want[0][:, 1, 2:])
    dy[T - 4, 1, ::2] = float("inf")
    _, dv, dh0 = nets.gate_scan_backward(f, v, want[0], dy, None)
    assert (dv[:T - 3, 1, ::2] == float("inf")).all() and (dh0[1, ::2] == float("inf")).all()
    assert torch.isfinite(dv[T - 3:]).all() and torch.isfinite(dv[:, 1, 1::2]).all() and torch.isfinite(dh0[0]).all()


@pytest.mark.parametrize("first", [30.0, 1000.0])
@pytest.mark.parametrize("B,S,C,G,dt", [(1, 65536, 8, 1, "fp32"), (1, 1 << 21, 4, 1, "fp32"), (1, 200000, 9, 3, "fp32"),
                                        (2, 70000, 16, 1, "bf16"), (3, 2000, 32, 4, "fp32"), (40, 300, 64, 8, "fp32")])
def test_norm_after_a_first_value_far_from_the_rest(B, S, C, G, dt, first):
    """One row a thousand deviations off at the start: the statistics are as exact as elsewhere."""
    torch, nets, types = _t()
    g = torch.Generator(device="cuda").manual_seed(33)
    x = torch.randn((B, S, C), device="cuda", generator=g)
    x[:, 0] *= first
    x = x.to(types[dt])
    y, mean, rstd = nets.group_norm(x, G)
    r = R.group_norm(_np(x), G, np.ones(C), np.zeros(C), 1e-5, "none")
    _within(mean, r[1], r[4])
    _within(rstd, r[2], r[5])
    _within(y, r[0], r[3], dt)


@pytest.mark.parametrize("layout", ["half", "odd"])
@pytest.mark.parametrize("T,N,D,dt", [(512, 300, 8, "bf16"), (300, 500, 1, "fp32"), (260, 400, 3, "fp16"), (200, 90, 40, "bf16"),
                                      (8192, 64, 1, "fp32"), (9001, 20, 3, "bf16")])
def test_recurrence_of_narrow_rows_apart(T, N, D, dt, layout):
    _check_scan(T, N, D, dt, layout, ends=0.01, seed=23)


@pytest.mark.parametrize("B,S,C,G", [(500, 300, 128, 1), (256, 1, 90, 9), (3, 5000, 64, 2), (70, 40, 48, 6)])
def test_a_workspace_sized_before_the_arrays_serves_any_alignment(B, S, C, G):
    torch, nets, types = _t()
    L, F = nets.lib(), nets._NORM
    n = B * S * C
    x, dy = (torch.randn(n + 8, device="cuda").to(torch.bfloat16) for _ in range(2))
    y, dx = (torch.empty(n + 8, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    mean, rstd = (torch.empty((B, G), device="cuda") for _ in range(2))
    dg, db = (torch.empty(C, device="cuda") for _ in range(2))

    def block(off, there=True):
        at = lambda t: (t.data_ptr() + 2 * off if there else 0, S * C, C)      # noqa: E731
        flat = [t.data_ptr() if there else 0 for t in (mean, rstd, dg, db)]
        return (F.size, 1, 2, 1e-5, B, S, C, G, *at(x), *at(y), *at(dy), *at(dx), 0, 0, *flat)
    need = [L.net_group_norm_workspace_bytes(F.pack(*block(0, False), 0, 0), back) for back in (0, 1)]
    ws = torch.empty(max(need) + 16, dtype=torch.uint8, device="cuda")
    for off in (0, 1, 2, 4, 7):
        for back, fn in enumerate((L.net_group_norm, L.net_group_norm_backward)):
            assert fn(F.pack(*block(off), ws.data_ptr(), need[back]), None) == 0, L.net_last_error()
        xs, ds = (t[off:off + n].view(B, S, C) for t in (x, dy))
        want = nets.group_norm(xs, G, act="silu")
        assert torch.equal(y[off:off + n].view(B, S, C), want[0]) and torch.equal(rstd, want[2])
        want = nets.group_norm_backward(xs, G, None, None, mean, rstd, ds, act="silu")
        assert torch.equal(dx[off:off + n].view(B, S, C), want[0]) and torch.equal(dg, want[1]) and torch.equal(db, want[2])


def test_arguments_of_a_wrong_kind():
    torch, nets, types = _t()
    from paper_2512_13359_gb300.auvenv import AUV_ERR_INVALID, AuvError
    x = torch.randn((4, 6, 8), device="cuda")
    stats = torch.zeros((4, 2), device="cuda")
    for bad in (lambda: nets.dropout(x, "0.5", 0, 0), lambda: nets.dropout(x, None, 0, 0),
                lambda: nets.dropout(x, 0.5, 1.5, 0), lambda: nets.dropout(x, 0.5, 0, None),
                lambda: nets.dropout(x, 0.5, 0, 0, residual=[1.0]), lambda: nets.group_norm(x, 2, eps="1"),
                lambda: nets.group_norm(x, 1 << 70), lambda: nets.group_norm(x, 2, [1.0] * 8),
                lambda: nets.group_norm(x, 2, y=3), lambda: nets.group_norm_backward(x, 2, None, None, stats, 1.0, x),
                lambda: nets.gate_scan(x, 1.0), lambda: nets.gate_scan(x, x, h0=0.0), lambda: nets.gate_scan(x, x, done=[0])):
        with pytest.raises(AuvError) as e:
            bad()
        assert e.value.code == AUV_ERR_INVALID, str(e.value)


@pytest.mark.parametrize("T,N,D,dt,layout", [
    (512, 1, 8192, "bf16", "flat"), (513, 5, 1031, "fp16", "odd"), (700, 40, 130, "fp32", "pad"), (1025, 3, 1700, "fp32", "flat"),
    (3000, 2, 600, "bf16", "half"), (1500, 37, 18, "fp16", "flat")])
def test_recurrence_in_rounds_of_blocks(T, N, D, dt, layout):
    """More steps than the blocks, or clusters of them, hold at a time."""
    _check_scan(T, N, D, dt, layout, ends=0.01, seed=21)


@pytest.mark.parametrize("T,N,D,dt,layout", [
    (45, 400, 256, "bf16", "flat"), (45, 400, 256, "fp32", "half"), (21, 3300, 30, "fp16", "flat"), (21, 3300, 30, "fp32", "flat"),
    (17, 1000, 100, "bf16", "pad"), (33, 3001, 36, "fp16", "half")])
def test_recurrence_of_many_channels_past_its_ring(T, N, D, dt, layout):
    _check_scan(T, N, D, dt, layout, ends=0.1, seed=22)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("B,S,C,G,layout", [
    (2, 9000, 18, 2, "flat"), (2, 9000, 18, 2, "half"),       # pieces of two groups, two wide
    (1, 20000, 24, 2, "pad"), (2, 6000, 12, 2, "flat"),       # and wider ones
    (2, 5000, 8, 8, "flat"), (1, 7000, 24, 8, "flat"),        # of many groups
    (1, 9000, 20, 1, "odd")])
def test_norm_by_chunks_whose_pieces_share_groups(B, S, C, G, layout, dt):
    _check_norm(B, S, C, G, dt, "silu", layout, seed=31)


@pytest.mark.parametrize("B,S,C,G,dt", [
    (200, 550, 80, 10, "bf16"), (200, 550, 80, 10, "fp32"),   # a last slab of fewer groups; a block an instance
    (200, 80, 64, 1, "bf16"), (170, 250, 72, 3, "fp16"),      # one block in either direction
    (3, 5000, 88, 11, "fp16"), (5, 900, 60, 5, "fp32")])      # fewer groups, in clusters
def test_norm_slabs(B, S, C, G, dt):
    _check_norm(B, S, C, G, dt, "silu", seed=32)
