"""The state space memory and the orthogonalised update without a GPU: refusals of argument blocks and tensors before a
device is touched; workspaces; the 64-bit reference (state_ref.py) against closed forms and differences."""
import numpy as np
import pytest

import state_ref as R
from nets_ref import act, sigmoid


@pytest.fixture(scope="module")
def nets():
    from paper_2512_13359_gb300 import build, nets
    build.build()
    nets.lib()
    return nets


def _blocks(nets):
    z = nets._NO_ROWS
    conv = [nets._CONV.size, 0, 0, 0, 2, 1, 4, 4, *(4 * z), *(11 * (0,)), 0]
    scan = [nets._SELECT.size, 0, 2, 1, 4, 8, 1, *(12 * z), *(14 * (0,)), 0]
    ortho = [nets._ORTHO.size, 0, 5, 1e-7, 3.4445, -4.775, 2.0315, 0, 1, 4, 4, *(2 * z), 0, 0]
    return {"net_causal_conv": (nets._CONV, conv), "net_causal_conv_backward": (nets._CONV, conv),
            "net_select_scan": (nets._SELECT, scan), "net_select_scan_backward": (nets._SELECT, scan),
            "net_orthogonalise": (nets._ORTHO, ortho)}


@pytest.mark.parametrize("fn,at,value,code,msg", [
    *[(fn, 0, 8, -1, "struct_size") for fn in ("net_causal_conv", "net_causal_conv_backward", "net_select_scan",
                                               "net_select_scan_backward", "net_orthogonalise")],
    *[(fn, 1, 3, -1, "dtype") for fn in ("net_causal_conv", "net_select_scan", "net_orthogonalise")],
    ("net_causal_conv", 2, 1, -1, "act"), ("net_causal_conv", 2, 9, -1, "act"), ("net_causal_conv", 3, 1, -1, "reserved"),
    ("net_causal_conv", 4, -1, -1, "negative"), ("net_causal_conv_backward", 6, -4, -1, "negative"),
    ("net_causal_conv", 7, 0, -1, "K < 1"), ("net_causal_conv", 7, 9, -6, "K past"), ("net_causal_conv", 5, 1 << 40, -6, "past"),
    ("net_causal_conv", 4, 1 << 40, -6, "past"), ("net_causal_conv", 1, 0, -1, "x is NULL"),
    ("net_select_scan", 2, -1, -1, "negative"), ("net_select_scan", 5, 0, -1, "S or G"), ("net_select_scan", 6, 0, -1, "S or G"),
    ("net_select_scan", 6, 3, -1, "multiple"), ("net_select_scan", 5, 129, -6, "S past"), ("net_select_scan", 3, 1 << 40, -6, "past"),
    ("net_select_scan", 2, 1 << 40, -6, "past"), ("net_select_scan_backward", 4, 1 << 30, -6, "past"),
    ("net_select_scan", 1, 0, -1, "x is NULL"), ("net_select_scan_backward", 1, 0, -1, "x is NULL"),
    ("net_orthogonalise", 2, 65, -1, "steps"), ("net_orthogonalise", 3, -1.0, -1, "eps"),
    ("net_orthogonalise", 3, float("nan"), -1, "eps"), ("net_orthogonalise", 3, float("inf"), -1, "eps"),
    ("net_orthogonalise", 4, float("nan"), -1, "coef"), ("net_orthogonalise", 4, 9.0, -6, "coef"),
    ("net_orthogonalise", 5, -700.0, -6, "coef"), ("net_orthogonalise", 7, 1, -1, "reserved"),
    ("net_orthogonalise", 8, -1, -1, "negative"), ("net_orthogonalise", 8, 65536, -6, "past"),
    ("net_orthogonalise", 9, (1 << 20) + 1, -6, "past"), ("net_orthogonalise", 1, 0, -1, "x is NULL"),
])
def test_bad_argument_blocks_are_rejected(nets, fn, at, value, code, msg):
    form, fields = _blocks(nets)[fn]
    fields[at] = value
    assert getattr(nets.lib(), fn)(form.pack(*fields), None) == code
    assert msg in nets.lib().net_last_error().decode()


def test_null_blocks_and_empty_calls(nets):
    for fn, (form, fields) in _blocks(nets).items():
        assert getattr(nets.lib(), fn)(None, None) == -1
        fields[10 if fn == "net_orthogonalise" else 6 if "conv" in fn else 4] = 0       # no channels: nothing to read or write
        # but gradients of B and C, which are sums over no channels then: zeros have to go somewhere
        assert getattr(nets.lib(), fn)(form.pack(*fields), None) == (-1 if fn == "net_select_scan_backward" else 0)
    assert nets.lib().net_causal_conv_workspace_bytes(None, 1) == 0
    assert nets.lib().net_select_scan_workspace_bytes(None, 1) == 0
    assert nets.lib().net_orthogonalise_workspace_bytes(None) == 0


def test_workspaces(nets):
    """Short sequences need none forward (the Python call does not ask), a convolution never; the gradients' weights do."""
    L = nets.lib()
    for N in (1, 3, 1000):
        for T in (1, 127, 128, 5000):
            for D, S, G in ((1, 1, 1), (250, 13, 1), (512, 16, 2)):
                form, f = _blocks(nets)["net_select_scan"]
                f[2:7] = T, N, D, S, G
                need = L.net_select_scan_workspace_bytes(form.pack(*f), 0)
                assert need == 0 or T >= 128
                assert L.net_select_scan_workspace_bytes(form.pack(*f), 1) >= 4 * D * (S + 2)
                form, f = _blocks(nets)["net_causal_conv"]
                f[4:7] = T, N, D
                assert L.net_causal_conv_workspace_bytes(form.pack(*f), 0) == 0
                assert L.net_causal_conv_workspace_bytes(form.pack(*f), 1) == 0         # no weight gradients asked for


@pytest.mark.parametrize("product,limit,msg", [(0, 20000, "product"), (15, 20000, "product"), (1, 0, "limit_us"), (14, 5000001, "limit_us"),
                                               (14, 20000, "x is NULL")])
def test_bad_limits_of_the_self_test_are_rejected(nets, product, limit, msg):
    form, fields = _blocks(nets)["net_orthogonalise"]
    assert nets.lib().net_orthogonalise_selftest_timeout(form.pack(*fields), product, limit, None) == -1
    assert msg in nets.lib().net_last_error().decode()
    assert nets.lib().net_orthogonalise_selftest_timeout(None, 1, 20000, None) == -1


def test_wrong_tensors_are_rejected(nets):
    import torch
    from paper_2512_13359_gb300.auvenv import AuvError
    x, w, A, b = torch.zeros(2, 3, 4), torch.zeros(4, 4), torch.zeros(4, 8), torch.zeros(2, 3, 8)
    for code, bad in ((-2, lambda: nets.causal_conv(x, w)), (-2, lambda: nets.select_scan(x, x, A, b, b)),
                      (-2, lambda: nets.orthogonalise(x)), (-1, lambda: nets.causal_conv(x.double(), w)),
                      (-1, lambda: nets.orthogonalise(x[0])), (-1, lambda: nets.select_scan(x[0], x, A, b, b)),
                      (-1, lambda: nets.orthogonalise([1.0]))):
        with pytest.raises(AuvError) as e:
            bad()
        assert e.value.code == code


# ------------------------------------------------------------ the reference itself
def _differences(loss, arrays, grads, rng, tol=1e-7):
    for k, (v, g) in enumerate(zip(arrays, grads)):
        if v is None:
            continue
        d, s = rng.normal(size=v.shape), 1e-6
        hi, lo = (loss(*[q + i * s * d if j == k else q for j, q in enumerate(arrays)]) for i in (1, -1))
        assert abs((hi - lo) / (2 * s) - (g * d).sum()) < tol * (1 + np.abs(g * d).sum()), k


@pytest.mark.parametrize("name", ["none", "silu"])
@pytest.mark.parametrize("T,K", [(1, 4), (2, 4), (9, 3), (9, 1), (5, 8)])
def test_reference_conv(T, K, name):
    rng = np.random.default_rng(T * 10 + K)
    N, D = 3, 2
    x, w, b, st = rng.normal(size=(T, N, D)), rng.normal(size=(K, D)), rng.normal(size=D), rng.normal(size=(K - 1, N, D))
    done, prev = rng.random((T, N)) < 0.3, np.array([1, 0, 0])
    dy, dn = rng.normal(size=(T, N, D)), rng.normal(size=(K - 1, N, D))
    # in one go and step by step, the state carried on
    y, new, _ = R.conv(x, w, b, st, done, prev, name)
    s, p = st, prev
    for t in range(T):
        yt, s, _ = R.conv(x[t:t + 1], w, b, s, None, p, name)
        assert np.allclose(yt[0], y[t], atol=1e-13)
        p = done[t]
    assert np.array_equal(s, new)
    loss = lambda x, w, b, st: (lambda y, n, _: (y * dy).sum() + (n * dn).sum())(*R.conv(x, w, b, st, done, prev, name))  # noqa: E731
    g = R.conv_backward(x, w, b, dy, st, done, prev, dn, name)
    _differences(loss, (x, w, b, st), g[:4], rng)


def test_reference_conv_closed_form():
    x = np.arange(1.0, 6.0)[:, None, None]
    w = np.array([[3.0], [2.0], [1.0]])                       # y[t] = x[t] + 2 x[t - 1] + 3 x[t - 2]
    y, new, _ = R.conv(x, w, np.zeros(1), None, None, None, "none")
    assert y[:, 0, 0].tolist() == [1, 4, 10, 16, 22] and new[:, 0, 0].tolist() == [4, 5]


@pytest.mark.parametrize("gated", [False, True])
def test_reference_scan(gated):
    rng = np.random.default_rng(5)
    T, N, D, S, G = 18, 2, 4, 3, 2
    r = lambda *s: rng.normal(size=s)                          # noqa: E731
    x, dt, B, C, gate = r(T, N, D), r(T, N, D), r(T, N, G * S), r(T, N, G * S), r(T, N, D) if gated else None
    A, skip, bias, h0, dhT, dy = -np.exp(r(D, S)), r(D), r(D), r(N, D, S), r(N, D, S), r(T, N, D)
    done, prev = rng.random((T, N)) < 0.15, np.array([0, 1])
    run = lambda x, dt, A, B, C, skip, bias, gate, h0: R.Scan(x, dt, A, B, C, skip, bias, gate, h0, done, prev)  # noqa: E731
    args = (x, dt, A, B, C, skip, bias, gate, h0)
    q = run(*args)
    # a channel by hand
    n, d, h = 1, 3, np.zeros(S)
    for t in range(T):
        if (prev[n] if t == 0 else done[t - 1, n]):
            h = np.zeros(S)
        elif t == 0:
            h = h0[n, d]
        e = np.log1p(np.exp(dt[t, n, d] + bias[d]))
        h = np.exp(e * A[d]) * h + e * x[t, n, d] * B[t, n, S:]
        y = (C[t, n, S:] * h).sum() + skip[d] * x[t, n, d]
        y = y * gate[t, n, d] * sigmoid(gate[t, n, d]) if gated else y
        assert abs(y - q.y[t, n, d]) < 1e-12
    assert np.allclose(h, q.hT[n, d]) and len(q.kept) == 2 and np.array_equal(q.kept[1], q.h[15])
    loss = lambda *a: (lambda s: (s.y * dy).sum() + (s.hT * dhT).sum())(run(*a))  # noqa: E731
    g = q.backward(dy, dhT)
    names = ("dx", "ddt", "dA", "dB", "dC", "dskip", "ddt_bias", "dgate", "dh0")
    _differences(loss, args, [g[k][0] if k in g else None for k in names], rng)


@pytest.mark.parametrize("M,N", [(3, 7), (7, 3), (4, 4), (1, 5)])
def test_reference_update_moves_singular_values(M, N):
    rng = np.random.default_rng(M)
    x, k = rng.normal(size=(M, N)), (3.4445, -4.775, 2.0315)
    y, _ = R.orthogonalise(x, 5, k, 0.0)
    u, v, w = np.linalg.svd(x, full_matrices=False)
    v = v / np.linalg.norm(v)
    for _ in range(5):
        v = k[0] * v + k[1] * v ** 3 + k[2] * v ** 5
    assert np.allclose(y, u * v @ w, atol=1e-12)


@pytest.mark.parametrize("M,N", R.RANK_ONE)
def test_bound_of_an_update_sees_a_lost_piece(M, N):
    """What the GPU's update of a matrix of one rank is held to is a third of what any of its products of pieces is to it."""
    assert np.isclose(R.rank_one_update(M, N, 1, R.RANK_ONE_COEF) * np.sqrt(M * N), 1.0, rtol=1e-6)
    for steps in (1, 2):
        bound = R.rank_one_bound(M, N, steps, R.RANK_ONE_COEF)
        whole = R.rank_one_update(M, N, steps, R.RANK_ONE_COEF) * np.sqrt(M * N) - 1
        assert abs(whole) < bound
        for lost in ("Phl", "Plh", "Qhl", "Qlh", "Xhl", "Xlh"):
            off = R.rank_one_update(M, N, steps, R.RANK_ONE_COEF, lost) * np.sqrt(M * N) - 1
            assert abs(off) > 3 * bound, (steps, lost, off / bound)


def test_reference_activation_is_the_operators():
    u = np.linspace(-20, 20, 41)
    assert np.allclose(act(u, "silu")[0], u / (1 + np.exp(-u)))
