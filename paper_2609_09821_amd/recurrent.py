"""A policy that remembers, trained on a context's rollouts.

    python -m paper_2609_09821_amd.recurrent [--envs N] [--steps K]

The rows of a rollout [T][envs] go through

    e = W_in obs + b_in,  u = rms_norm(e),  (gate, x) = W_g u + b_g,
    s = gated_scan(gate, x),  h = e + W_o s,  mean = W_out rms_norm(h) + b_out.

All four products are in 8 bits (e4m3 in blocks of 128 that share a power of two; weights in blocks
of 128 x 128), the scan's state is that of the envs and is cleared where an episode ends.  Training
keeps, of a rollout, the transposed 8-bit inputs of the products, the residual stream in bf16 and
the scan's states at each sixteenth step.  Run as a program it imitates the actions of a context's
own policy, rollout by rollout as the envs move on, and prints the loss.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as im

EPS = 1e-6


class RecurrentPolicy:
    """Float32 master weights, and the products' weights in 8 bits as they lie and transposed."""

    LAYERS = ("in", "gate", "out", "mean")

    def __init__(self, obs_dim, hidden, actions, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.dims = (obs_dim, hidden, actions)
        f = dict(device=device)
        sizes = dict(zip(self.LAYERS, ((hidden, obs_dim), (2 * hidden, hidden), (hidden, hidden),
                                       (actions, hidden))))
        self.w = {k: torch.randn(o, i, generator=g, **f) * i ** -0.5 for k, (o, i) in sizes.items()}
        self.b = {k: torch.zeros(sizes[k][0], **f) for k in ("in", "gate", "mean")}
        self.b["gate"][:hidden] = 2.0          # remembers for some ten steps
        self.gamma = [torch.ones(hidden, **f) for _ in range(2)]
        self.w8 = {k: im.Block8.empty(o, i, im.IM_BLOCK8, device) for k, (o, i) in sizes.items()}
        self.w8t = {k: im.Block8.empty(i, o, im.IM_BLOCK8, device) for k, (o, i) in sizes.items()}
        self.refresh()

    def params(self):
        return [*self.w.values(), *self.b.values(), *self.gamma]

    def refresh(self):
        """The 8-bit weights from the master weights."""
        for k, w in self.w.items():
            im.block8_store(w, self.w8[k], self.w8t[k])


class Rollout:
    """Buffers and workspaces of a policy on T steps of n envs; `state` [n][hidden] is the
    envs' memory, which forward() takes from step to step and from rollout to rollout."""

    def __init__(self, policy, T, n, train=False, device="cuda"):
        d, h, a = policy.dims
        self.T, self.n, M = T, n, T * n

        def rows(width, dtype=torch.bfloat16):
            return torch.zeros(M, -(-width // 8) * 8, dtype=dtype, device=device)[:, :width]

        f = dict(device=device)
        self.x, self.e, self.u, self.z = rows(d), rows(h), rows(h), rows(2 * h)
        self.s, self.r, self.h, self.v = rows(h), rows(h), rows(h), rows(h)
        self.mean = torch.zeros(M, a, **f)
        self.rstd = [torch.zeros(M, **f) for _ in range(2)]
        widths = {"in": d, "gate": h, "out": h, "mean": h}
        self.x8 = {k: im.Block8.empty(M, w, device=device) for k, w in widths.items()}
        self.state = torch.zeros(n, h, **f)
        self.ws_scan = im.gated_scan_workspace(T, n, h)
        if not train:
            self.x8t = dict.fromkeys(widths)
            self.keep = None
            return
        self.x8t = {k: im.Block8.empty(w, M, device=device) for k, w in widths.items()}
        self.keep = torch.zeros(-(-T // im.IM_SCAN_KEEP), n, h, **f)
        self.dmean, self.dv, self.dh, self.ds = rows(a), rows(h), rows(h), rows(h)
        self.dz, self.du, self.de = rows(2 * h), rows(h), rows(h)
        self.grads = [torch.zeros_like(p) for p in policy.params()]
        self.ws = {k: im.linear8_grad_workspace(M, w.shape[1], w.shape[0])
                   for k, w in policy.w.items()}
        self.ws_norm = im.rms_norm_grad_workspace(M, h)

    def steps(self, t):
        """[T][n][..] of a matrix of the rollout's rows."""
        return t.unflatten(0, (self.T, self.n))

    def halves(self, t):
        """Gates and values, the halves of the product's rows."""
        t, h = self.steps(t), t.shape[1] // 2
        return t[..., :h], t[..., h:]


def forward(policy, ro, terminated=None, truncated=None):
    """Means of ro.x's rows (into ro.mean) from ro.state, which becomes that after the last step;
    terminated, truncated: [T][n], where an env's episode ends with a step (either may be None)."""
    p = policy

    def store(x, k):
        im.block8_store(x, ro.x8[k], ro.x8t[k])

    store(ro.x, "in")
    im.linear8(ro.x8["in"], p.w8["in"], p.b["in"], ro.e)
    im.rms_norm(ro.e, p.gamma[0], ro.u, ro.rstd[0], EPS)
    store(ro.u, "gate")
    im.linear8(ro.x8["gate"], p.w8["gate"], p.b["gate"], ro.z)
    im.gated_scan(*ro.halves(ro.z), ro.steps(ro.s), ro.state, ro.state, ro.keep, terminated, truncated,
                  ro.ws_scan)
    store(ro.s, "out")
    im.linear8(ro.x8["out"], p.w8["out"], None, ro.r)
    im.rms_norm(ro.r, p.gamma[1], ro.v, ro.rstd[1], EPS, residual=ro.e, h=ro.h)
    store(ro.v, "mean")
    im.linear8(ro.x8["mean"], p.w8["mean"], p.b["mean"], ro.mean)
    return ro.mean


def backward(policy, ro, terminated=None, truncated=None):
    """Gradients of the policy's params() for ro.dmean within the rollout (the state that it
    began with counts as given)."""
    p = policy
    dw_in, dw_gate, dw_out, dw_mean, db_in, db_gate, db_mean, dg0, dg1 = ro.grads
    im.linear8_grad(ro.dmean, ro.x8t["mean"], p.w8t["mean"], ro.dv, dw_mean, db_mean,
                    workspace=ro.ws["mean"])
    im.rms_norm_grad(ro.dv, ro.h, p.gamma[1], ro.rstd[1], ro.dh, dg1, workspace=ro.ws_norm)
    im.linear8_grad(ro.dh, ro.x8t["out"], p.w8t["out"], ro.ds, dw_out, workspace=ro.ws["out"])
    im.gated_scan_grad(ro.steps(ro.ds), *ro.halves(ro.z), ro.keep, *ro.halves(ro.dz),
                       terminated=terminated, truncated=truncated, workspace=ro.ws_scan)
    im.linear8_grad(ro.dz, ro.x8t["gate"], p.w8t["gate"], ro.du, dw_gate, db_gate,
                    workspace=ro.ws["gate"])
    im.rms_norm_grad(ro.du, ro.e, p.gamma[0], ro.rstd[0], ro.de, dg0, dh=ro.dh, workspace=ro.ws_norm)
    im.linear8_grad(ro.de, ro.x8t["in"], None, None, dw_in, db_in, workspace=ro.ws["in"])
    return ro.grads


def imitate(envs=1024, steps=20, T=16, workload=4, seed=1, log=print):
    """Trains a RecurrentPolicy on the means of a context's policy (a synthetic workload's, by
    default the S24 humanoid on 16 clips), a rollout of T steps at a time; returns its losses."""
    from . import synth

    desc = synth.make_world(workload, n_envs=envs)
    ctx = im.Context(desc, max_envs=envs, critic=False)
    bufs = ctx.buffers(envs)
    store = im.RolloutStorage(ctx, envs, T, ld=bufs.ld)
    ctx.reset_envs(bufs)
    store.obs[0].copy_(bufs.obs)
    policy = RecurrentPolicy(ctx.info.obs_dim, 256, ctx.info.action_dim, seed)
    ro = Rollout(policy, T, envs, train=True)
    ends = store.terminated[:, :envs], store.truncated[:, :envs]
    opt = torch.optim.Adam(policy.params(), lr=2e-3)
    losses = []
    for step in range(steps):
        for t in range(T):
            ctx.policy_act(store.obs[t], bufs.env_n, envs, store.mean[t], store.action[t])
            ctx.standin_physics(bufs, desc["sigma_joint"], desc["sigma_vel"])
            ctx.env_step_fused(store.env_bufs(bufs, t))
        ro.steps(ro.x).copy_(store.obs[:T, :, :envs].transpose(1, 2))
        diff = forward(policy, ro, *ends) - store.mean[:, :envs].reshape(T * envs, -1)
        ro.dmean.copy_(diff * (2.0 / diff.numel()))
        for p, g in zip(policy.params(), backward(policy, ro, *ends)):
            p.grad = g
        opt.step()
        policy.refresh()
        store.obs[0].copy_(store.obs[T])
        losses.append(float(diff.square().mean()))
        if step % 5 == 0 or step + 1 == steps:
            log("rollout %3d: loss %.5f" % (step, losses[-1]))
    ctx.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--envs", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    imitate(a.envs, a.steps)
