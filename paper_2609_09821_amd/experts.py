"""A policy with a layer of experts, trained on a context's rollout observations.

    python -m paper_2609_09821_amd.experts [--envs N] [--steps K]

One network for many clips: the rows of a batch (envs) are grouped by their clip's
expert, normed, and go through two layers whose weights go by the expert:

    u = layer_norm(obs),  h = relu(W1_e u + b1_e),  mean = W2_e h + b2_e.

Training keeps the three activations in 8 bits and no others: the gradients of the
weights, the ReLU's mask and the norm's gradient are taken from them.  The mask is that
of the kept h: a hidden unit of at most half a step, about one in a hundred of those
that are active, passes no gradient back in that pass.  Run as a
program it imitates the actions of a context's own policy on the envs' observations,
step by step as the envs move on, and prints the loss.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as im


class ExpertPolicy:
    """Two layers of `n_experts` experts behind a layer norm: float32 master weights,
    bfloat16 copies for the products, rows padded to 16 bytes."""

    def __init__(self, n_experts, obs_dim, hidden, actions, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.E, self.dims = n_experts, (obs_dim, hidden, actions)
        f = dict(device=device)
        self.gamma, self.beta = torch.ones(obs_dim, **f), torch.zeros(obs_dim, **f)
        self.w, self.b, self.w16 = [], [], []
        for i, o in ((obs_dim, hidden), (hidden, actions)):
            self.w.append(torch.randn(n_experts, o, i, generator=g, **f) * i ** -0.5)
            self.b.append(torch.zeros(n_experts, o, **f))
            wide = torch.zeros(n_experts, o, -(-i // 8) * 8, dtype=torch.bfloat16, **f)
            self.w16.append(wide[:, :, :i])
        self.refresh()

    def params(self):
        return [self.gamma, self.beta, *self.w, *self.b]

    def refresh(self):
        """The bfloat16 copies from the master weights."""
        for w, w16 in zip(self.w, self.w16):
            w16.copy_(w)


class Batch:
    """Buffers and workspaces of a policy on batches of n rows."""

    def __init__(self, policy, n, device="cuda"):
        d, h, a = policy.dims
        E = policy.E

        def rows(width, dtype=torch.bfloat16):
            return torch.zeros(n, -(-width // 8) * 8, dtype=dtype, device=device)[:, :width]

        f = dict(device=device)
        self.n = n
        self.offsets = torch.zeros(E + 1, dtype=torch.int32, **f)
        self.order = torch.zeros(n, dtype=torch.int32, **f)
        self.x, self.u, self.h = rows(d), rows(d), rows(h)
        self.mean = torch.zeros(n, a, **f)
        self.row_mean, self.row_rstd = torch.zeros(n, **f), torch.zeros(n, **f)
        self.keep_x, self.keep_u, self.keep_h = (im.Checkpoint.empty(n, -(-w // 16) * 16, device)
                                                 for w in (d, d, h))
        for c, w in ((self.keep_x, d), (self.keep_u, d), (self.keep_h, h)):
            c.q, c.scale = c.q[:, :w], c.scale[:, :-(-w // 32)]
        self.dmean, self.dh, self.du = rows(a), rows(h), rows(d)
        self.grads = [torch.zeros_like(p) for p in policy.params()]
        self.ws_group = im.group_rows_workspace(n, E)
        self.ws = [im.expert_linear_grad_workspace(n, E, d, h),
                   im.expert_linear_grad_workspace(n, E, h, a)]
        self.ws_norm = im.layer_norm_grad_workspace(n, d)


def forward(policy, batch, expert, train=False):
    """Means of batch.x's rows (into batch.mean) by their experts (int32 [n]; a row whose
    expert is none of the policy's gets zeros); train: keeps the activations in 8 bits."""
    b, p = batch, policy
    im.group_rows(expert, b.offsets, b.order, b.ws_group)
    im.layer_norm(b.x, p.gamma, p.beta, b.u, b.row_mean, b.row_rstd,
                  checkpoint=b.keep_x if train else None)
    im.expert_linear(b.u, p.w16[0], p.b[0], b.offsets, b.order, b.h, relu=True)
    im.expert_linear(b.h, p.w16[1], p.b[1], b.offsets, b.order, b.mean)
    if train:
        im.checkpoint_store(b.u, b.keep_u)
        im.checkpoint_store(b.h, b.keep_h)
    return b.mean


def backward(policy, batch):
    """Gradients of the policy's params() for batch.dmean, from the kept activations."""
    b, p = batch, policy
    dgamma, dbeta, dw1, dw2, db1, db2 = b.grads
    im.expert_linear_grad(b.dmean, b.keep_h, p.w16[1], b.offsets, b.order, b.dh, dw2, db2,
                          relu_x=True, workspace=b.ws[1])
    im.expert_linear_grad(b.dh, b.keep_u, p.w16[0], b.offsets, b.order, b.du, dw1, db1,
                          workspace=b.ws[0])
    im.layer_norm_grad(b.du, b.keep_x, p.gamma, b.row_mean, b.row_rstd, None, dgamma, dbeta,
                       workspace=b.ws_norm)
    return b.grads


def imitate(envs=4096, steps=60, workload=4, seed=1, log=print):
    """Trains an ExpertPolicy on the means of a context's policy (a synthetic workload's,
    by default the S24 humanoid on 16 clips); returns its losses."""
    from . import synth

    desc = synth.make_world(workload, n_envs=envs)
    ctx = im.Context(desc, max_envs=envs, critic=False)
    bufs = ctx.buffers(envs)
    ctx.reset_envs(bufs)
    A = ctx.info.action_dim
    teacher = [torch.zeros(envs, A, device="cuda") for _ in range(2)]   # mean, action
    policy = ExpertPolicy(ctx.info.n_clips, ctx.info.obs_dim, 256, A, seed)
    batch = Batch(policy, envs)
    opt = torch.optim.Adam(policy.params(), lr=2e-3)
    losses = []
    for step in range(steps):
        ctx.policy_act(bufs.obs, bufs.env_n, envs, *teacher)
        batch.x.copy_(bufs.obs[:, :envs].t())
        # an env's clip changes with its resets: the rows are grouped anew each step
        mean = forward(policy, batch, bufs.env_clip[:envs], train=True)
        diff = mean - teacher[0]
        batch.dmean.copy_(diff * (2.0 / diff.numel()))
        for p, g in zip(policy.params(), backward(policy, batch)):
            p.grad = g
        opt.step()
        policy.refresh()
        losses.append(float(diff.square().mean()))
        if step % 10 == 0 or step + 1 == steps:
            log("step %3d: loss %.5f" % (step, losses[-1]))
        ctx.standin_physics(bufs, desc["sigma_joint"], desc["sigma_vel"])
        ctx.env_step_fused(bufs)
    ctx.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--envs", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    imitate(a.envs, a.steps)
