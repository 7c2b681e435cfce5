"""A critic with memory, trained on rollouts with a hidden water current.

The current, the mass and the buoyancy of an episode (domain randomisation) are not in the observation: what a state is
worth depends on them, so a critic gains from remembering the episode.  This one has the network operators of
paper_2512_13359_gb300.nets between two dense products (auvenv.gemm), in the order of DroQ's critic (dropout, then layer
norm, then ReLU) with a gated recurrence in front:

    z = obs W^T         [T, N, 2D]    gate and value halves
    h = gate_scan       [T, N, D]     episode ends cut the state; the state goes on from one rollout to the next
    u = dropout(h)                    one mask for all steps of an update
    o = relu(layer norm(u))
    V = o w + b         [T, N]

Its loss is the mean squared distance to the TD(lambda) targets of env_gae; all gradients are the operators' own.

    python examples/memory_critic.py [--envs 4096] [--steps 64] [--rollouts 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2512_13359_gb300 import auvenv, nets, workloads as W  # noqa: E402


class MemoryCritic:
    """fp32 weights on the current device; Adam."""

    def __init__(self, obs_dim: int, width: int, p: float = 0.05, seed: int = 0, lr: float = 1e-2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.obs_dim, self.width, self.p, self.seed, self.lr = obs_dim, width, p, seed, lr
        self.draw = self.steps = 0           # masks drawn, updates made: a pass that only values draws a mask too
        self.w = dict(z=torch.randn(2 * width, obs_dim, device="cuda", generator=g) * obs_dim ** -0.5,
                      gamma=torch.ones(width, device="cuda"), beta=torch.zeros(width, device="cuda"),
                      v=torch.randn(1, width, device="cuda", generator=g) * width ** -0.5,
                      b=torch.zeros(1, device="cuda"))
        self.w["z"][:width] *= 0.1                       # gates start half open, whatever the observation
        self.m1 = {k: torch.zeros_like(x) for k, x in self.w.items()}
        self.m2 = {k: torch.zeros_like(x) for k, x in self.w.items()}
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda")

    def _gemm(self, M, N, K, A, lda, a_mn, B, ldb, b_mn, C, ldc):
        auvenv.gemm("fp32", M, N, K, A, lda, a_mn, B, ldb, b_mn, C, ldc, status=self.status)
        return C

    def step(self, obs, state, ended):
        """Values [N] of one control step's observations [N, obs_dim], without dropout; state [N, D] in place; ended:
        the flags of the step before."""
        n, d = obs.shape[0], self.width
        z = self._gemm(n, 2 * d, self.obs_dim, obs, self.obs_dim, False, self.w["z"], self.obs_dim, False,
                       torch.empty((1, n, 2 * d), device="cuda"), 2 * d)
        h, _ = nets.gate_scan(z[..., :d], z[..., d:], state, done_prev=ended, hT=state)
        o, _, _ = nets.group_norm(h.view(n, 1, d), 1, self.w["gamma"], self.w["beta"], act="relu")
        v = self._gemm(n, 1, d, o, d, False, self.w["v"], d, False, torch.empty((n, 1), device="cuda"), 1)
        return v[:, 0] + self.w["b"]

    def forward(self, obs, state, done, ended):
        """Values [T, N] of observations [T, N, obs_dim] and what backward needs; hT is the state after the last step."""
        T, N, _ = obs.shape
        d, rows = self.width, obs.shape[0] * obs.shape[1]
        self.draw += 1
        z = self._gemm(rows, 2 * d, self.obs_dim, obs, self.obs_dim, False, self.w["z"], self.obs_dim, False,
                       torch.empty((T, N, 2 * d), device="cuda"), 2 * d)
        h, hT = nets.gate_scan(z[..., :d], z[..., d:], state, done=done, done_prev=ended)
        u = nets.dropout(h, self.p, self.seed, self.draw, shared=True)
        o, mean, rstd = nets.group_norm(u.view(rows, 1, d), 1, self.w["gamma"], self.w["beta"], act="relu")
        v = self._gemm(rows, 1, d, o, d, False, self.w["v"], d, False, torch.empty((rows, 1), device="cuda"), 1)
        values = v.view(T, N) + self.w["b"]
        return values, dict(obs=obs, state=state, done=done, ended=ended, z=z, h=h, u=u, o=o, mean=mean, rstd=rstd, hT=hT)

    def backward(self, dvalues, s):
        """Gradients of the weights from the values' [T, N]."""
        T, N = dvalues.shape
        d, rows = self.width, T * N
        dv = dvalues.reshape(rows, 1).contiguous()
        g = dict(b=dvalues.sum().view(1))
        g["v"] = self._gemm(1, d, rows, dv, 1, True, s["o"], d, True, torch.empty((1, d), device="cuda"), d)
        do = self._gemm(rows, d, 1, dv, 1, False, self.w["v"], d, True, torch.empty((rows, 1, d), device="cuda"), d)
        du, g["gamma"], g["beta"] = nets.group_norm_backward(s["u"].view(rows, 1, d), 1, self.w["gamma"], self.w["beta"],
                                                             s["mean"], s["rstd"], do, act="relu")
        dh = nets.dropout(du.view(T, N, d), self.p, self.seed, self.draw, shared=True, y=du.view(T, N, d))
        z, dz = s["z"], torch.empty_like(s["z"])
        nets.gate_scan_backward(z[..., :d], z[..., d:], s["h"], dh, s["state"], done=s["done"], done_prev=s["ended"],
                                df=dz[..., :d], dv=dz[..., d:])
        g["z"] = self._gemm(2 * d, self.obs_dim, rows, dz, 2 * d, True, s["obs"], self.obs_dim, True,
                            torch.empty((2 * d, self.obs_dim), device="cuda"), self.obs_dim)
        return g

    def update(self, obs, targets, state, done, ended):
        """One Adam step towards the targets [T, N]; returns the loss (on the device) and the state after."""
        values, s = self.forward(obs, state, done, ended)
        err = values - targets
        g = self.backward(err / err.numel(), s)
        self.steps += 1
        c1, c2 = 1 - 0.9 ** self.steps, 1 - 0.99 ** self.steps
        for k, w in self.w.items():
            self.m1[k].lerp_(g[k].view_as(w), 0.1)
            self.m2[k].lerp_(g[k].view_as(w) ** 2, 0.01)
            w -= self.lr * (self.m1[k] / c1) / ((self.m2[k] / c2).sqrt() + 1e-8)
        return 0.5 * (err ** 2).mean(), s["hT"]


def train(n_envs: int, steps: int, rollouts: int, epochs: int = 4, width: int = 64, report=print):
    """Rollouts of a random policy in randomised currents; each is learned from `epochs` times.  Returns the losses."""
    w = W.workload("ppo_65536", n_envs=n_envs, episode_len=100)
    env = auvenv.Env(w)
    env.set_weights(W.policy_weights(w), W.value_weights(w))
    env.reset()
    critic = MemoryCritic(W.OBS_DIM, width)
    traj = env.alloc_traj(steps, keys=("obs", "act", "rew", "done"))
    state = torch.zeros((n_envs, width), device="cuda")
    ended = torch.zeros(n_envs, dtype=torch.uint8, device="cuda")
    last_obs = torch.empty((W.OBS_DIM, n_envs), device="cuda")
    losses = []
    for it in range(rollouts):
        env.rollout(steps, traj)
        env.observe(last_obs)
        obs = traj["obs"].permute(0, 2, 1).contiguous()                 # [T, N, 18] rows
        values, s = critic.forward(obs, state, traj["done"], ended)
        end_state = s["hT"].clone()
        bootstrap = critic.step(last_obs.t().contiguous(), s["hT"], traj["done"][-1])
        adv, targets = torch.empty_like(values), torch.empty_like(values)
        traj["rew"] *= 0.03                                             # values of order one: 1 - discount
        env.gae(traj["rew"], traj["done"], values.contiguous(), bootstrap, 0.97, 0.9, adv, targets)
        for _ in range(epochs):
            loss, _ = critic.update(obs, targets, state, traj["done"], ended)
            losses.append(loss)
        state, ended = end_state, traj["done"][-1].clone()
        report(f"rollout {it}: loss {float(losses[-epochs]):.4f} -> {float(losses[-1]):.4f}")
    assert env.status().code == 0 and int(critic.status[0]) == 0
    return torch.stack(losses)


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    a.add_argument("--envs", type=int, default=4096)
    a.add_argument("--steps", type=int, default=64)
    a.add_argument("--rollouts", type=int, default=8)
    args = a.parse_args()
    train(args.envs, args.steps, args.rollouts)
