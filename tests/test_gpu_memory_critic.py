"""The network operators together, as examples/memory_critic.py uses them: the critic's values and gradients against the
same network in 64 bits with torch's own differentiation, its steps against its sequence, and a short training."""
import os
import sys

import numpy as np
import pytest

import nets_ref as R
from parity_util import need_gpu

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _critic(torch, width=24, p=0.25):
    import memory_critic as M
    c = M.MemoryCritic(18, width, p=p, seed=5)
    g = torch.Generator(device="cuda").manual_seed(9)
    c.w["gamma"] += 0.2 * torch.randn(width, device="cuda", generator=g)
    c.w["beta"] += 0.2 * torch.randn(width, device="cuda", generator=g)
    return c, g


def test_gradients_of_the_whole_network():
    torch = need_gpu()
    c, g = _critic(torch)
    T, N, d = 12, 37, c.width
    obs = torch.randn((T, N, 18), device="cuda", generator=g)
    state = torch.randn((N, d), device="cuda", generator=g)
    done = (torch.rand((T, N), device="cuda", generator=g) < 0.1).to(torch.uint8)
    ended = (torch.rand((N,), device="cuda", generator=g) < 0.2).to(torch.uint8)
    values, s = c.forward(obs, state, done, ended)
    dvalues = torch.randn((T, N), device="cuda", generator=g) / (T * N)
    got = c.backward(dvalues, s)
    w = {k: x.double().requires_grad_() for k, x in c.w.items()}
    z = obs.double() @ w["z"].t()
    keep = torch.from_numpy(R.dropout_keep(N * d, c.p, c.seed, c.draw)).cuda().view(N, d)
    h, outs = state.double(), []
    for t in range(T):
        e = (ended if t == 0 else done[t - 1]).bool()[:, None]
        a = torch.sigmoid(z[t, :, :d])
        h = a * torch.where(e, torch.zeros_like(h), h) + (1 - a) * z[t, :, d:]
        u = h * keep
        m, v = u.mean(1, keepdim=True), u.var(1, unbiased=False, keepdim=True)
        outs.append(torch.relu((u - m) / torch.sqrt(v + 1e-5) * w["gamma"] + w["beta"]) @ w["v"].t())
    ref = torch.stack(outs)[..., 0] + w["b"]
    # fp32 against 64 bits over a handful of operators: some 1e-6 of the largest value, 2e-5 leaves room for sums' order
    assert (values - ref).abs().max() <= 2e-5 * ref.abs().max()
    want = torch.autograd.grad(ref, [w[k] for k in c.w], dvalues.double())
    for k, x in zip(c.w, want):
        assert (got[k].view_as(x) - x).abs().max() <= 2e-5 * x.abs().max(), k


def test_steps_follow_the_sequence():
    torch = need_gpu()
    c, g = _critic(torch, p=0.0)
    T, N = 9, 50
    obs = torch.randn((T, N, 18), device="cuda", generator=g)
    state = torch.randn((N, c.width), device="cuda", generator=g)
    done = (torch.rand((T, N), device="cuda", generator=g) < 0.2).to(torch.uint8)
    ended = torch.zeros(N, dtype=torch.uint8, device="cuda")
    values, s = c.forward(obs, state, done, ended)
    h = state.clone()
    for t in range(T):
        v = c.step(obs[t].contiguous(), h, ended if t == 0 else done[t - 1])
        assert (v - values[t]).abs().max() <= 1e-5 * values.abs().max()
    assert (h - s["hT"]).abs().max() <= 1e-5


def test_training_lowers_the_loss():
    need_gpu()
    import memory_critic as M
    losses = M.train(512, 40, 6, report=lambda *_: None).cpu().numpy()
    assert np.isfinite(losses).all() and losses[-4:].mean() < 0.7 * losses[:4].mean()
