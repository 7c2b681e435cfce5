"""The network operators on a GPU where their plans change and where fp32 ends, against the 64-bit reference
(nets_ref.py)."""
import numpy as np
import pytest

import nets_ref as R
from test_gpu_nets import DT, _np, _t, _within

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
