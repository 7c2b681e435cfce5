"""The updates of examples/memory_critic.py."""
import os
import sys

import pytest

from parity_util import need_gpu

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _inputs(torch, T=6, N=20, width=24):
    import memory_critic as M
    c = M.MemoryCritic(18, width, seed=5)
    g = torch.Generator(device="cuda").manual_seed(9)
    obs = torch.randn((T, N, 18), device="cuda", generator=g)
    state = torch.zeros((N, width), device="cuda")
    done = torch.zeros((T, N), dtype=torch.uint8, device="cuda")
    return c, obs, torch.randn((T, N), device="cuda", generator=g), state, done, done[0]


def test_outputs_overlap_no_other_array(monkeypatch):
    torch = need_gpu()
    from paper_2512_13359_gb300 import nets
    c, obs, targets, state, done, ended = _inputs(torch)
    seen = []
    call = nets.group_norm_backward

    def watch(x, groups, gamma, beta, mean, rstd, dy, **out):
        ins = {t.data_ptr() for t in (x, gamma, beta, mean, rstd, dy) if t is not None}
        seen.append(all(t.data_ptr() not in ins for t in out.values() if isinstance(t, torch.Tensor)))
        return call(x, groups, gamma, beta, mean, rstd, dy, **out)
    monkeypatch.setattr(nets, "group_norm_backward", watch)
    c.update(obs, targets, state, done, ended)
    assert seen and all(seen)


def test_the_first_update_is_adams_first_step():
    """Whatever was valued before: with both moments corrected for one step, m1 / sqrt(m2) is the gradient's sign and
    each weight moves by the rate."""
    torch = need_gpu()
    c, obs, targets, state, done, ended = _inputs(torch)
    for _ in range(3):
        c.forward(obs, state, done, ended)
    before = {k: w.clone() for k, w in c.w.items()}
    c.update(obs, targets, state, done, ended)
    for k, w in c.w.items():
        # gradients are some 1e-2, of which 1e-8 in the denominator takes 1e-6, and weights of order 1 round to 1e-7
        moved = (w - before[k]).abs().max()
        assert abs(moved - c.lr) <= 1e-3 * c.lr, (k, float(moved))
