"""The network operators without a GPU: the library exports what include/auvnet.h declares and rejects bad argument
blocks before touching a device; the 64-bit reference (nets_ref.py) against closed forms and differences."""
import os
import re

import numpy as np
import pytest

import nets_ref as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def nets():
    from paper_2512_13359_gb300 import build, nets
    build.build()
    nets.lib()
    return nets


def test_exports_what_the_header_declares(nets):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "auvnet.h")).read(), flags=re.S)
    names = re.findall(r"^\s*(?:const\s+)?\w+\s*\**\s*(net_\w+)\s*\(", text, flags=re.M)
    assert sorted(names) == sorted(nets.EXPORTED)
    for n in names:
        assert hasattr(nets.lib(), n)


def _blocks(nets):
    z = nets._NO_ROWS
    scan = [nets._SCAN.size, 0, 1, 1, 1, *(6 * z), *(7 * (0,)), 0]
    norm = [nets._NORM.size, 0, 0, 1e-5, 1, 1, 4, 2, *(4 * z), *(7 * (0,)), 0]
    drop = [nets._DROP.size, 0, 0, 0, 1, 1, 1, *(3 * z), 0.5, 0, 0]
    return {"net_gate_scan": (nets._SCAN, scan), "net_gate_scan_backward": (nets._SCAN, scan),
            "net_group_norm": (nets._NORM, norm), "net_group_norm_backward": (nets._NORM, norm),
            "net_dropout": (nets._DROP, drop)}


@pytest.mark.parametrize("fn,at,value,code,msg", [
    *[(fn, 0, 8, -1, "struct_size") for fn in ("net_gate_scan", "net_gate_scan_backward", "net_group_norm",
                                               "net_group_norm_backward", "net_dropout")],
    ("net_gate_scan", 1, 3, -1, "dtype"), ("net_group_norm", 1, 3, -1, "dtype"), ("net_dropout", 1, 3, -1, "dtype"),
    ("net_gate_scan", 2, -1, -1, "negative"), ("net_gate_scan_backward", 4, -1, -1, "negative"),
    ("net_gate_scan", 3, 1 << 40, -6, "past"), ("net_gate_scan", 2, 1 << 60, -6, "past"),
    ("net_gate_scan", 1, 0, -1, "f is NULL"),
    ("net_group_norm", 2, 4, -1, "act"), ("net_group_norm", 3, -1.0, -1, "eps"),
    ("net_group_norm", 3, float("nan"), -1, "eps"), ("net_group_norm", 7, 0, -1, "G < 1"),
    ("net_group_norm", 7, 3, -1, "multiple"), ("net_group_norm_backward", 6, -4, -1, "negative"),
    ("net_group_norm", 6, 1 << 25, -6, "past"), ("net_group_norm", 4, 1 << 51, -6, "past"),
    ("net_group_norm", 1, 0, -1, "x is NULL"),
    ("net_dropout", 2, 2, -1, "shared"), ("net_dropout", 3, 1, -1, "reserved"), ("net_dropout", 16, 1.5, -1, "p outside"),
    ("net_dropout", 16, float("nan"), -1, "p outside"), ("net_dropout", 5, 1 << 51, -6, "past"),
    ("net_dropout", 6, -2, -1, "negative"), ("net_dropout", 1, 0, -1, "x is NULL"),
])
def test_bad_argument_blocks_are_rejected(nets, fn, at, value, code, msg):
    form, fields = _blocks(nets)[fn]
    fields[at] = value
    assert getattr(nets.lib(), fn)(form.pack(*fields), None) == code
    assert msg in nets.lib().net_last_error().decode()


def test_null_blocks_and_empty_calls(nets):
    for fn, (form, fields) in _blocks(nets).items():
        assert getattr(nets.lib(), fn)(None, None) == -1
        n = {"net_dropout": 6, "net_group_norm": 6, "net_group_norm_backward": 6}.get(fn, 4)
        fields[n] = 0                                            # no channels: nothing to read or write
        assert getattr(nets.lib(), fn)(form.pack(*fields), None) == 0
    assert nets.lib().net_group_norm_workspace_bytes(None, 0) == 0
    assert nets.lib().net_gate_scan_workspace_bytes(None, 0) == 0


def test_wrong_tensors_are_rejected(nets):
    import torch
    from paper_2512_13359_gb300.auvenv import AuvError
    x = torch.zeros(2, 3, 4)
    for bad in (lambda: nets.gate_scan(x, x), lambda: nets.group_norm(x, 2), lambda: nets.dropout(x, 0.5, 0, 0)):
        with pytest.raises(AuvError) as e:                       # host memory
            bad()
        assert e.value.code == -2
    for bad in (lambda: nets.gate_scan(x[0], x[0]), lambda: nets.group_norm(x.double(), 2),
                lambda: nets.dropout([1.0], 0.5, 0, 0)):
        with pytest.raises(AuvError) as e:
            bad()
        assert e.value.code == -1


# ------------------------------------------------------------ the reference itself
def test_reference_recurrence_closed_forms():
    T, N, D = 6, 2, 3
    f, v = np.full((T, N, D), 0.7), np.full((T, N, D), 2.0)
    h0 = np.ones((N, D))
    y, hT, _, _ = R.gate_scan(f, v, h0, None, None)
    a = R.sigmoid(0.7)
    k = np.arange(1, T + 1)[:, None, None]
    assert np.allclose(y, a ** k + 2.0 * (1 - a ** k), atol=1e-14) and np.array_equal(hT, y[-1])
    done = np.zeros((T, N)); done[2, 1] = 1
    z, _, _, _ = R.gate_scan(f, v, h0, done, np.array([1, 0]))
    assert np.allclose(z[0, 0], 2 * (1 - a)) and np.allclose(z[0, 1], y[0, 1])      # done_prev
    assert np.allclose(z[3, 1], 2 * (1 - a)) and np.allclose(z[2, 1], y[2, 1])      # done


@pytest.mark.parametrize("ends", [False, True])
def test_reference_recurrence_gradient_by_differences(ends):
    rng = np.random.default_rng(3)
    T, N, D = 7, 2, 3
    f, v, dy = (rng.normal(size=(T, N, D)) for _ in range(3))
    h0, dhT = (rng.normal(size=(N, D)) for _ in range(2))
    done = (rng.random((T, N)) < 0.3) if ends else None
    prev = np.array([1, 0]) if ends else None
    loss = lambda f, v, h0: (lambda y, hT: (y * dy).sum() + (hT * dhT).sum())(*R.gate_scan(f, v, h0, done, prev)[:2])  # noqa: E731
    y = R.gate_scan(f, v, h0, done, prev)[0]
    grads = R.gate_scan_backward(f, v, y, dy, h0, done, prev, dhT)[:3]
    for k in range(3):
        d = rng.normal(size=(f, v, h0)[k].shape)
        e = 1e-6
        hi, lo = (loss(*[q + s * e * d if i == k else q for i, q in enumerate((f, v, h0))]) for s in (1, -1))
        assert abs((hi - lo) / (2 * e) - (grads[k] * d).sum()) < 1e-8 * (1 + np.abs(grads[k] * d).sum())


@pytest.mark.parametrize("name", R.ACTS)
def test_reference_norm_gradient_by_differences(name):
    rng = np.random.default_rng(4)
    B, S, C, G = 2, 3, 6, 2
    x, dy = rng.normal(size=(B, S, C)), rng.normal(size=(B, S, C))
    p = [x, 1 + 0.2 * rng.normal(size=C), 0.2 * rng.normal(size=C)]
    loss = lambda x, g, b: (R.group_norm(x, G, g, b, 1e-5, name)[0] * dy).sum()  # noqa: E731
    _, mean, rstd, *_ = R.group_norm(*p[:1], G, *p[1:], 1e-5, name)
    grads = R.group_norm_backward(x, G, p[1], p[2], mean, rstd, dy, name)[:3]
    for k in range(3):
        d = rng.normal(size=p[k].shape)
        e = 1e-6
        hi, lo = (loss(*[q + s * e * d if i == k else q for i, q in enumerate(p)]) for s in (1, -1))
        assert abs((hi - lo) / (2 * e) - (grads[k] * d).sum()) < 1e-7 * (1 + np.abs(grads[k] * d).sum())


def test_reference_generator_known_answers():
    # Salmon et al.'s published vectors of Philox4x32-10
    assert [hex(q) for q in R.philox(0, 0, 0, 0, 0, 0)[0]] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    m = 0xFFFFFFFF
    assert [hex(q) for q in R.philox(m, m, m, m, m, m)[0]] == ["0x408f276d", "0x41c83b0e", "0xa20bc7c6", "0x6d5451fd"]
    k = R.dropout_keep(80000, 0.25, 5, 6)
    assert set(np.unique(k)) == {0.0, 65536 / 49152} and abs((k == 0).mean() - 0.25) < 4 * np.sqrt(0.1875 / 80000)
    assert (R.dropout_keep(100, 0.0, 1, 2) == 1).all() and (R.dropout_keep(100, 1.0, 1, 2) == 0).all()
