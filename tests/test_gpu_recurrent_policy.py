"""The policy that remembers: its run as a whole stage by stage against 64 bits, its gradients,
steps one at a time, graphs, streams, and training."""
import numpy as np
import pytest
import torch

from paper_2609_09821_amd import binding as im
from paper_2609_09821_amd import recurrent
from tests import recurrent_oracle as O

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8 * 1.01           # a rounding to bf16
FAST = 7 * 2.0 ** -13             # 8-bit products to bf16: what eight products' sum may lose of its terms


def _np(t):
    return t.detach().float().cpu().double().numpy()


def _held(b):
    return O.unpack8(b.q.view(torch.uint8).cpu().numpy(), b.scale.cpu().numpy(), b.d, b.rows)


def _within(got, want, tol):
    bad = np.abs(got - want) > tol
    assert not bad.any(), (bad.sum(), np.abs(got - want)[bad].max())


def _filled(T, n, dims, seed):
    p = recurrent.RecurrentPolicy(*dims, seed=seed)
    ro = recurrent.Rollout(p, T, n, train=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ro.x.copy_(torch.randn(T * n, dims[0], device="cuda", generator=g))
    ro.state.copy_(torch.randn(n, dims[1], device="cuda", generator=g))
    ends = (torch.rand(2, T, n, device="cuda", generator=g) < 0.1).to(torch.uint8)
    ro.dmean.copy_(1e-3 * torch.randn(T * n, dims[2], device="cuda", generator=g))
    for t in p.gamma:
        t.add_(0.2 * torch.randn(t.shape, device="cuda", generator=g))
    return p, ro, ends


@pytest.mark.parametrize("T,n,dims", [(1, 1, (226, 64, 28)), (20, 7, (361, 96, 69)), (40, 40, (70, 136, 9))])
def test_the_whole_stage_by_stage(T, n, dims):
    """Each stage against 64 bits from the values that it was given, so that every difference is
    that stage's own: the bounds of the operators' own tests."""
    p, ro, ends = _filled(T, n, dims, T)
    state0 = _np(ro.state)
    recurrent.forward(p, ro, *ends)
    grads = recurrent.backward(p, ro, *ends)
    M, H = T * n, dims[1]
    end = (ends[0] | ends[1]).cpu().numpy() != 0

    def product(x8, k, y, half):
        xv, wv = _held(x8), _held(p.w8[k])
        bias = _np(p.b[k]) if k in p.b else 0.0
        want, mass = xv @ wv.T + bias, np.abs(xv) @ np.abs(wv).T
        tol = (xv.shape[1] + 2) * 2 * O.U32 * (mass + np.abs(bias)) + (FAST * mass if half else 0)
        _within(_np(y), want, tol + (HALF * (np.abs(want) + tol) if half else O.U32 * np.abs(want)))

    stored = {"in": ro.x, "gate": ro.u, "out": ro.s, "mean": ro.v}
    for k, x in stored.items():
        np.testing.assert_array_equal(_held(ro.x8[k]), O.unpack8(*O.pack8(_np(x)), x.shape[1]))
        np.testing.assert_array_equal(_held(ro.x8t[k]), O.unpack8(*O.pack8(_np(x).T.copy()), M))
        np.testing.assert_array_equal(_held(p.w8[k]).T, _held(p.w8t[k]))
    product(ro.x8["in"], "in", ro.e, True)
    product(ro.x8["gate"], "gate", ro.z, True)
    product(ro.x8["out"], "out", ro.r, True)
    product(ro.x8["mean"], "mean", ro.mean, False)
    h, rstd, v = O.rms_norm(_np(ro.r), _np(ro.e), _np(p.gamma[1]), recurrent.EPS)
    size = np.abs(_np(ro.r)) + np.abs(_np(ro.e))
    _within(_np(ro.h), h, HALF * size)
    _within(_np(ro.v), v, HALF * np.abs(v) + 64 * O.U32 * size * rstd[:, None] * np.abs(_np(p.gamma[1])))
    gate, x = (_np(t) for t in ro.halves(ro.z))
    s, before, last, es, ebefore, elast = O.scan(gate, x, end, state0)
    _within(_np(ro.steps(ro.s)), s, es + HALF * (np.abs(s) + es))
    _within(_np(ro.state), last, elast)
    _within(_np(ro.keep), before[::16], ebefore[::16])

    def product_grad(dy, k, dx, dw, db):
        m = _np(dy)
        cols, xv = O.unpack8(*O.pack8(m.T.copy()), M), _held(ro.x8t[k])
        _within(_np(dw), cols @ xv.T, (M + 2) * 2 * O.U32 * (np.abs(cols) @ np.abs(xv).T))
        if db is not None:
            _within(_np(db), m.sum(0), 130 * O.U32 * np.abs(m).sum(0))
        if dx is not None:
            rows, wv = O.unpack8(*O.pack8(m), m.shape[1]), _held(p.w8t[k])
            want, mass = rows @ wv.T, np.abs(rows) @ np.abs(wv).T
            tol = ((m.shape[1] + 2) * 2 * O.U32 + FAST) * mass
            _within(_np(dx), want, tol + HALF * (np.abs(want) + tol))

    dw_in, dw_gate, dw_out, dw_mean, db_in, db_gate, db_mean, dg0, dg1 = grads
    product_grad(ro.dmean, "mean", ro.dv, dw_mean, db_mean)
    product_grad(ro.dh, "out", ro.ds, dw_out, None)
    product_grad(ro.dz, "gate", ro.du, dw_gate, db_gate)
    product_grad(ro.de, "in", None, dw_in, db_in)

    def norm_grad(dy, h, dh, k, dx, dg):
        dy, h, gamma, rstd = _np(dy), _np(h), _np(p.gamma[k]), _np(ro.rstd[k])
        want, dgw = O.rms_norm_grad(dy, h, None if dh is None else _np(dh), gamma, rstd)
        u, gg = h * rstd[:, None], dy * gamma
        mag = rstd[:, None] * (np.abs(gg) + np.abs(u) * np.abs(gg * u).mean(1, keepdims=True))
        mag = mag + (0 if dh is None else np.abs(_np(dh)))
        _within(_np(dx), want, 28 * O.U32 * mag + HALF * np.abs(want))
        _within(_np(dg), dgw, (M + 8) * O.U32 * np.abs(dy * u).sum(0))

    norm_grad(ro.dv, ro.h, None, 1, ro.dh, dg1)
    norm_grad(ro.du, ro.e, ro.dh, 0, ro.de, dg0)
    dgate, dx, _, eg, ex, _ = O.scan_grad(_np(ro.steps(ro.ds)), gate, x, end, before, ebefore, np.zeros((n, H)))
    got = [_np(t) for t in ro.halves(ro.dz)]
    _within(got[0], dgate, eg + HALF * (np.abs(dgate) + eg))
    _within(got[1], dx, ex + HALF * (np.abs(dx) + ex))


def test_steps_one_at_a_time():
    """Served step by step, each env's memory in place, the policy says what it says of the rollout,
    to the bit: a row's sums go by its own values in any batch that takes the same tiles."""
    p, ro, ends = _filled(12, 9, (100, 64, 20), 3)
    state0 = ro.state.clone()
    whole = recurrent.forward(p, ro, *ends).clone()
    one = recurrent.Rollout(p, 1, 9)
    one.state.copy_(state0)
    x = ro.steps(ro.x)
    for t in range(12):
        one.x.copy_(x[t])
        mean = recurrent.forward(p, one, ends[0, t:t + 1], ends[1, t:t + 1])
        assert torch.equal(mean, whole[t * 9:(t + 1) * 9])
    assert torch.equal(one.state, ro.state)


def _snapshot(ro, grads=True):
    return [t.clone() for t in (ro.mean, ro.state, ro.h, *(ro.grads if grads else ()))]


def test_graphs_and_streams():
    """Forward and backward captured as two graphs with workspaces of their own, replayed in turn with
    eager work between, and the same calls on a side stream, give the eager bits."""
    runs = []
    for seed in (1, 2):
        p, ro, ends = _filled(33, 20, (90, 72, 12), seed)
        state0 = ro.state.clone()

        def step(p=p, ro=ro, ends=ends, state0=state0):
            ro.state.copy_(state0)
            recurrent.forward(p, ro, *ends)
            recurrent.backward(p, ro, *ends)

        step()
        torch.cuda.synchronize()
        runs.append((step, ro, _snapshot(ro)))
    graphs = []
    for step, ro, _ in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    scratch = torch.zeros(1 << 20, device="cuda")
    for k in range(4):
        for _, ro, _ in runs:
            for t in (ro.mean, ro.h, *ro.grads):
                t.fill_(7.0)
        for g in graphs if k % 2 else graphs[::-1]:
            g.replay()
        scratch.add_(1.0).sum()
        torch.cuda.synchronize()
        for _, ro, want in runs:
            assert all(torch.equal(a, b) for a, b in zip(_snapshot(ro), want)), k
    side = [torch.cuda.Stream() for _ in runs]
    for _, ro, _ in runs:
        for t in (ro.mean, ro.h, *ro.grads):
            t.fill_(7.0)
    torch.cuda.synchronize()
    for (step, _, _), s in zip(runs, side):
        with torch.cuda.stream(s):
            step()
    torch.cuda.synchronize()
    for _, ro, want in runs:
        assert all(torch.equal(a, b) for a, b in zip(_snapshot(ro), want))


def test_a_stream_that_is_not_current():
    """`stream` and no workspace: the calls' own scratch memory is of that stream."""
    s = torch.cuda.Stream()
    g = torch.randn(5000, 2, 6, device="cuda")
    h, want = torch.zeros_like(g), torch.zeros_like(g)
    im.gated_scan(g, g, want)
    torch.cuda.synchronize()
    im.gated_scan(g, g, h, stream=s)
    dy, x = torch.randn(700, 40, device="cuda"), torch.randn(700, 24, device="cuda")
    torch.cuda.synchronize()
    xt = im.Block8.empty(24, 700)
    im.block8_store(x, None, xt, stream=s)
    dw, db, dw2, db2 = (torch.zeros(*z, device="cuda") for z in ((40, 24), (40,), (40, 24), (40,)))
    torch.cuda.synchronize()
    im.linear8_grad(dy, xt, None, None, dw, db, stream=s)
    im.linear8_grad(dy, xt, None, None, dw2, db2)
    torch.cuda.synchronize()
    assert torch.equal(h, want) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_imitation_runs():
    """Rollouts of moving envs, their episodes' ends and the updates between them."""
    said = []
    losses = recurrent.imitate(envs=192, steps=3, T=18, log=said.append)
    assert len(losses) == 3 and all(np.isfinite(losses)) and said
