"""Layers of experts on the GPU against their formulas in float64.

Tolerances (u = 2^-24, fp32's unit roundoff; bf16's is 2^-9):
* whole numbers (group_rows, the checkpoint's q and scale) and restored values: equal;
* a product's sum of K terms: products of two bf16 values are exact in fp32, so the
  error of summing them in any order, each addition rounded or cut off, is at most
  2 K u sum |terms|; a bf16 result adds 2^-8 of itself (one rounding);
* layer norm: fp32 sums over a row of at most 8192 values in 64 lanes or more are
  at most 8 * 4 additions in a lane and 8 across lanes deep: 48 u relative to the sum
  of magnitudes, 64 with the operations around them;
* dgamma and dbeta: at most ROWS additions in a lane (the tests' rows are few) plus
  16 across lanes, wavefronts and blocks.
"""
import math

import numpy as np
import pytest
import torch

from paper_2609_09821_amd import binding as im

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8
DEV = "cuda"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _wide(x, pad):
    """x as a view of rows that are `pad` wider, the padding NaN (or -1)."""
    fill = float("nan") if x.is_floating_point() else -1
    w = torch.full((x.shape[0], x.shape[1] + pad), fill, dtype=x.dtype, device=DEV) \
        if x.dtype != torch.uint8 else \
        torch.full((x.shape[0], x.shape[1] + pad), 77, dtype=x.dtype, device=DEV)
    w[:, :x.shape[1]] = x
    return w[:, :x.shape[1]]


def _out(n, d, pad, dtype):
    return _wide(torch.zeros((n, d), dtype=dtype, device=DEV), pad)


def _pad_kept(t):
    """The padding of a view made by _wide is as it was."""
    if t.dim() != 2 or t.shape[0] == 0 or t.stride(0) == t.shape[1]:
        return
    full = t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1))[:, t.shape[1]:]
    assert bool(torch.isnan(full).all() if full.is_floating_point() else
                (full == (77 if t.dtype == torch.uint8 else -1)).all())


def _within(got, want, tol, what=""):
    d = (got.double() - want).abs()
    bad = ~(d <= tol)
    assert not bool(bad.any()), "%s: %d of %d out of tolerance, worst %.3g of it" % (
        what, int(bad.sum()), bad.numel(), float((d / tol.clamp(min=1e-300)).max()))


# ------------------------------------------------------------------ group_rows
def _group_ref(e, E):
    e = e.cpu().numpy()
    k = np.where((e >= 0) & (e < E), e, E)
    rows = np.argsort(k, kind="stable")
    off = np.searchsorted(k[rows], np.arange(E + 1))
    return off, rows


@pytest.mark.parametrize("n,E", [(0, 3), (1, 1), (1, 1024), (63, 2), (64, 8), (65, 7), (1024, 64),
                                 (1025, 65), (5000, 1), (70001, 63), (300000, 64), (40000, 1024),
                                 (1 << 20, 17)])
@pytest.mark.parametrize("form", ["even", "none", "one", "wild"])
def test_group_rows(n, E, form):
    g = _gen(n + E)
    e = torch.randint(0, E, (n,), device=DEV, dtype=torch.int32, generator=g)
    if form == "none":
        e = torch.full_like(e, -1)
    elif form == "one":
        e = torch.full_like(e, E - 1)
    elif form == "wild":
        w = torch.tensor([-1, E, 2 ** 31 - 1, -2 ** 31, E + 63], device=DEV, dtype=torch.int32)
        pick = torch.randint(0, 10, (n,), device=DEV, generator=g)
        e = torch.where(pick < 5, w[pick.clamp(max=4)], e)
    off = torch.full((E + 1,), -7, device=DEV, dtype=torch.int32)
    rows = torch.full((n,), -7, device=DEV, dtype=torch.int32)
    im.group_rows(e, off, rows)
    o, r = _group_ref(e, E)
    assert np.array_equal(off.cpu().numpy(), o) and np.array_equal(rows.cpu().numpy(), r)


# ------------------------------------------------------------------ checkpoints
def _ckpt_ref(x):
    """(q, scale, restored) in float64 from the definition."""
    x = x.double().cpu().numpy()
    n, d = x.shape
    nb = -(-d // 32)
    b = np.zeros((n, nb * 32))
    b[:, :d] = x
    b = b.reshape(n, nb, 32)
    bad = ~np.isfinite(b).all(2)
    b = np.where(bad[:, :, None], 0.0, b)
    top = np.abs(b).max(2)
    e = np.where(top > 0, np.frexp(top)[1] - 1, -127).clip(-127, 127)
    up = (np.round(top * 2.0 ** (6.0 - e)) > 127) & (e < 127)
    e = e + up
    q = np.round(b * 2.0 ** (6.0 - e)[:, :, None]).clip(-127, 127)
    v = q * 2.0 ** (e - 6.0)[:, :, None]
    v[bad] = np.nan
    scale = np.where(bad, 255, e + 127)
    return q.reshape(n, nb * 32)[:, :d], scale, v.reshape(n, nb * 32)[:, :d], bad


def _check_ckpt(x, ck):
    q, scale, v, bad = _ckpt_ref(x)
    n, d = x.shape
    assert np.array_equal(ck.scale.cpu().numpy(), scale)
    keep = ~np.repeat(bad, 32, axis=1)[:, :d]
    assert np.array_equal(ck.q.cpu().numpy()[keep], q[keep])
    return v


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,pad", [(0, 5, 0), (1, 1, 0), (3, 7, 0), (5, 32, 0), (2, 33, 1),
                                     (130, 69, 3), (1000, 361, 0), (257, 538, 6), (64, 1024, 0),
                                     (3, 9001, 0)])
def test_checkpoint(n, d, pad, dtype):
    g = _gen(n * 31 + d)
    x = torch.randn(n, d, device=DEV, generator=g) * \
        torch.exp2(torch.randint(-40, 40, (n, 1), device=DEV, generator=g).float())
    x = _wide(x.to(dtype), pad)
    ck = im.Checkpoint(_out(n, d, pad, torch.int8), _out(n, -(-d // 32), pad, torch.uint8))
    im.checkpoint_store(x, ck)
    v = _check_ckpt(x, ck)
    _pad_kept(ck.q), _pad_kept(ck.scale)
    for back in (torch.float32, torch.bfloat16):
        y = _out(n, d, pad, back)
        im.checkpoint_load(ck, y)
        assert np.array_equal(y.double().cpu().numpy(), v)
        _pad_kept(y)
    # half a step from the original, and the step the smallest that holds the block (its
    # largest magnitude is at least 63.75 steps: 127.5 halves of them)
    xd = x.double().cpu().numpy()
    step = 2.0 ** (ck.scale.cpu().numpy().astype(np.float64) - 133)
    for c in range(0, d, 32):
        top = np.abs(xd[:, c:c + 32]).max(1, initial=0.0)
        s = step[:, c // 32]
        assert (np.abs(xd[:, c:c + 32] - v[:, c:c + 32]).max(1, initial=0.0) <= s / 2).all()
        assert (top >= 63.75 * s).all() and (top <= 127.5 * s).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_checkpoint_extremes(dtype):
    """Zeros, subnormals, the largest values, infinities and NaN, in blocks of their own."""
    big = torch.finfo(dtype).max
    tiny = 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149
    x = torch.randn(14, 64, device=DEV, generator=_gen(5)).to(dtype)
    x[0] = 0
    x[1, :32] = 0
    x[2, 3] = float("inf")
    x[3, 40] = float("nan")
    x[4, :] = -float("inf")
    x[5, 7] = big
    x[6, 7] = -big
    x[7] = tiny
    x[8, :32] = torch.arange(32, device=DEV) * tiny
    x[9] = 2.0 ** -126
    x[10] = x[10] * 2.0 ** -126
    x[11, 0] = 127.5 / 64
    x[12, 0] = 255 / 128.0
    x[13, 0] = -127.4 / 64
    ck = im.Checkpoint.empty(14, 64)
    im.checkpoint_store(x, ck)
    v = _check_ckpt(x, ck)
    for back in (torch.float32, torch.bfloat16):
        y = torch.zeros(14, 64, dtype=back, device=DEV)
        im.checkpoint_load(ck, y)
        assert np.array_equal(y.double().cpu().numpy(), v, equal_nan=True)


# ------------------------------------------------------------------ layer norm
NORM_SHAPES = [(1, 1, 0), (1, 1024, 0), (3, 2, 1), (70, 28, 0), (33, 33, 3), (513, 69, 0),
               (100, 226, 2), (257, 361, 0), (64, 512, 0), (129, 538, 0), (65, 1024, 8),
               (31, 1101, 3), (17, 2048, 0), (9, 2049, 0), (5, 4097, 1), (3, 8192, 0)]


def _norm_inputs(n, d, pad, dtype, seed):
    g = _gen(seed)
    x = torch.randn(n, d, device=DEV, generator=g) * (0.2 + torch.rand(d, device=DEV, generator=g))
    x = x + 3.0 * torch.randn(d, device=DEV, generator=g)
    gamma = torch.randn(d, device=DEV, generator=g)
    beta = torch.randn(d, device=DEV, generator=g)
    return _wide(x.to(dtype), pad), gamma, beta, g


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,pad", NORM_SHAPES)
def test_layer_norm(n, d, pad, dtype):
    x, gamma, beta, _ = _norm_inputs(n, d, pad, dtype, n + 7 * d)
    eps = 1e-3
    xd = x.double()
    mean = xd.mean(1)
    var = (xd - mean[:, None]).square().mean(1)
    rstd = (var + eps) ** -0.5
    h = (xd - mean[:, None]) * rstd[:, None]
    size = xd.abs().mean(1)
    for ga, be in ((gamma, beta), (None, beta), (gamma, None), (None, None)):
        y = _out(n, d, pad, dtype)
        m, r = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        ck = im.Checkpoint(_out(n, d, pad, torch.int8), _out(n, -(-d // 32), pad, torch.uint8))
        im.layer_norm(x, ga, be, y, m, r, eps=eps, checkpoint=ck)
        gd = torch.ones(d, device=DEV).double() if ga is None else ga.double()
        bd = torch.zeros(d, device=DEV).double() if be is None else be.double()
        want = h * gd + bd
        _within(m, mean, 64 * U * size, "mean")
        # a shift of the mean by delta adds delta^2 to the variance, 2 delta / n |x - mean| to
        # its error's first order (which cancels); var is relative to itself + eps
        drstd = 64 * U * rstd + 64 * U * size * rstd * rstd
        _within(r, rstd, drstd, "rstd")
        tol = gd.abs() * (rstd * 64 * U * size)[:, None] + (gd * h).abs() * \
            (64 * U + 64 * U * size * rstd)[:, None] + 4 * U * want.abs() + \
            4 * U * (gd * h).abs() + 4 * U * gd.abs() * (xd.abs() * rstd[:, None])
        if dtype == torch.bfloat16:
            tol = tol + BF * want.abs()
        _within(y, want, tol, "y")
        _pad_kept(y)
        _check_ckpt(x, ck)
        _pad_kept(ck.q), _pad_kept(ck.scale)
    # without statistics, in place
    y2 = x.clone() if pad == 0 else _wide(x.contiguous(), pad)
    im.layer_norm(y2, gamma, beta, y2, eps=eps)
    y = _out(n, d, pad, dtype)
    im.layer_norm(x, gamma, beta, y, eps=eps)
    assert torch.equal(y, y2)


def _ngrad_ref(dy, x, gamma, mean, rstd):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    h = (x - mean) * rstd
    g = dy * gamma.double()
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    size = rstd * (g.abs() + g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0), size, (dy * h).abs().sum(0), dy.abs().sum(0), h


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,pad", NORM_SHAPES + [(5000, 64, 0), (3001, 361, 7)])
def test_layer_norm_grad(n, d, pad, dtype, kept):
    x, gamma, beta, g = _norm_inputs(n, d, pad, dtype, n + 3 * d)
    dy = _wide(torch.randn(n, d, device=DEV, generator=g).to(dtype), pad)
    y = _out(n, d, pad, dtype)
    m, r = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    ck = im.Checkpoint(_out(n, d, pad, torch.int8), _out(n, -(-d // 32), pad, torch.uint8))
    im.layer_norm(x, gamma, beta, y, m, r, eps=1e-2, checkpoint=ck)
    xin = torch.from_numpy(_ckpt_ref(x)[2]).to(DEV) if kept else x
    want, dgam, dbet, size, sg, sb, _ = _ngrad_ref(dy, xin, gamma, m, r)
    dx = _out(n, d, pad, dtype)
    dg, db = torch.full((d,), 9.0, device=DEV), torch.full((d,), 9.0, device=DEV)
    src = ck if kept else x
    im.layer_norm_grad(dy, src, gamma, m, r, dx, dg, db)
    tol = 64 * U * size
    if dtype == torch.bfloat16:
        tol = tol + BF * want.abs()
    _within(dx, want, tol + 1e-300, "dx")
    _pad_kept(dx)
    # x - mean is rounded once, times rstd once more: 2 u of |h|
    rows = 64 + 16
    _within(dg, dgam, rows * U * sg + 1e-300, "dgamma")
    _within(db, dbet, rows * U * sb + 1e-300, "dbeta")
    # each output alone, and twice the same bits
    dg2, db2, dx2 = torch.zeros_like(dg), torch.zeros_like(db), _out(n, d, pad, dtype)
    im.layer_norm_grad(dy, src, gamma, m, r, dgamma=dg2)
    im.layer_norm_grad(dy, src, gamma, m, r, dbeta=db2)
    im.layer_norm_grad(dy, src, gamma, m, r, dx=dx2)
    assert torch.equal(dg, dg2) and torch.equal(db, db2) and torch.equal(dx, dx2)
    # in place over dy; no gamma is gamma 1
    dy2 = _wide(dy.contiguous(), pad)
    im.layer_norm_grad(dy2, src, gamma, m, r, dx=dy2)
    assert torch.equal(dy2, dx)
    im.layer_norm_grad(dy, src, None, m, r, dx=dx)
    im.layer_norm_grad(dy, src, torch.ones(d, device=DEV), m, r, dx=dx2)
    assert torch.equal(dx, dx2)


def test_layer_norm_grad_no_rows_and_nan_row():
    d = 40
    dg, db = torch.full((d,), 3.0, device=DEV), torch.full((d,), 3.0, device=DEV)
    e = torch.zeros(0, d, device=DEV)
    z = torch.zeros(0, device=DEV)
    im.layer_norm_grad(e, e, None, z, z, e, dg, db)
    assert not dg.any() and not db.any()
    x = torch.randn(20, d, device=DEV, generator=_gen(1))
    x[7, 3] = float("nan")
    x[9, 5] = float("inf")
    y = torch.zeros_like(x)
    m, r = torch.zeros(20, device=DEV), torch.zeros(20, device=DEV)
    im.layer_norm(x, None, None, y, m, r)
    dx = torch.zeros_like(x)
    im.layer_norm_grad(torch.ones_like(x), x, None, m, r, dx)
    for t in (y, dx):
        bad = torch.isnan(t).any(1)
        assert bad.nonzero().flatten().tolist() == [7, 9]


def test_layer_norm_grad_against_differences():
    """dx, dgamma, dbeta against central differences of the float64 forward.  With steps of
    1e-4 the differences' own error is below 1e-7 of the sums' sizes; fp32 gradients add
    64 u of theirs."""
    n, d, eps = 6, 45, 1e-2
    x, gamma, beta, g = _norm_inputs(n, d, 0, torch.float32, 3)
    dy = torch.randn(n, d, device=DEV, generator=g)
    y, m, r = torch.zeros_like(x), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    im.layer_norm(x, gamma, beta, y, m, r, eps=eps)
    dx, dg, db = torch.zeros_like(x), torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    im.layer_norm_grad(dy, x, gamma, m, r, dx, dg, db)

    def loss(x, ga, be):
        mu = x.mean(1, keepdim=True)
        return ((x - mu) * ((x - mu).square().mean(1, keepdim=True) + eps) ** -0.5 * ga + be).mul(dy.double()).sum()

    args = [x.double(), gamma.double(), beta.double()]
    for k, grad in enumerate((dx, dg, db)):
        for t in range(4):
            v = torch.randn(args[k].shape, device=DEV, generator=g, dtype=torch.float64)
            s = 1e-4
            up, dn = list(args), list(args)
            up[k], dn[k] = args[k] + s * v, args[k] - s * v
            diff = float((loss(*up) - loss(*dn)) / (2 * s))
            dot = float((grad.double() * v).sum())
            assert abs(diff - dot) <= 1e-5 * float((grad.double() * v).abs().sum() + v.abs().sum())


# ------------------------------------------------------------------ expert layers
def _layer(n, E, din, dout, pad, seed, form="even", order=True):
    g = _gen(seed)
    e = torch.randint(0, E, (n,), device=DEV, dtype=torch.int32, generator=g)
    if form == "one":
        e = torch.full_like(e, E // 2)
    elif form == "holes":
        e = torch.where(torch.rand(n, device=DEV, generator=g) < 0.3, torch.full_like(e, -1), e)
        e = torch.where(e == E // 2, torch.full_like(e, -1), e)
    elif form == "none":
        e = torch.full_like(e, -1)
    if not order:
        e = torch.sort(torch.where(e < 0, torch.full_like(e, E), e)).values
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    rows = torch.zeros(n, dtype=torch.int32, device=DEV)
    im.group_rows(e, off, rows)
    x = _wide(torch.randn(n, din, device=DEV, generator=g).bfloat16(), pad)
    w = _wide((torch.randn(E * dout, din, device=DEV, generator=g) / math.sqrt(din)).bfloat16(), pad)
    return e, off, (rows if order else None), x, w.unflatten(0, (E, dout)), \
        torch.randn(E, dout, device=DEV, generator=g), g


def _by_expert(e, E):
    e = e.cpu()
    return [torch.nonzero(e == k).flatten().to(DEV) for k in range(E)]


LAYERS = [  # n, E, in, out, pad, form
    (1, 1, 1, 1, 0, "even"), (1, 5, 361, 1024, 7, "even"), (7, 3, 28, 69, 0, "even"),
    (64, 8, 226, 130, 6, "even"), (300, 4, 64, 64, 0, "holes"), (513, 2, 361, 257, 0, "even"),
    (1000, 16, 128, 96, 0, "holes"), (700, 70, 65, 128, 7, "even"), (900, 5, 512, 69, 0, "one"),
    (257, 3, 1000, 129, 8, "even"), (260, 4, 33, 40, 0, "none"), (4000, 3, 72, 200, 0, "holes"),
]


@pytest.mark.parametrize("n,E,din,dout,pad,form", LAYERS)
def test_expert_linear(n, E, din, dout, pad, form):
    for order in (True, False):
        e, off, rows, x, w, b, _ = _layer(n, E, din, dout, pad, n + din, form, order)
        for relu, bias, dt in ((False, b, torch.bfloat16), (True, b, torch.float32),
                               (True, None, torch.bfloat16), (False, None, torch.float32)):
            want = torch.zeros(n, dout, device=DEV, dtype=torch.float64)
            size = torch.zeros_like(want)
            for k, r in enumerate(_by_expert(e, E)):
                want[r] = x[r].double() @ w[k].double().t()
                size[r] = x[r].double().abs() @ w[k].double().abs().t()
                if bias is not None:
                    want[r] += bias[k].double()
                    size[r] += bias[k].double().abs()
            if relu:
                want = want.clamp(min=0)
            y = _out(n, dout, pad, dt)
            y.fill_(5.0)
            im.expert_linear(x, w, bias, off, rows, y, relu=relu)
            tol = 2 * (din + 1) * U * size
            if dt == torch.bfloat16:
                tol = tol + BF * want.abs()
            _within(y, want, tol, "y")
            _pad_kept(y)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("n,E,din,dout,pad,form", LAYERS)
def test_expert_linear_grad(n, E, din, dout, pad, form, kept):
    for order, relu in ((True, False), (False, True), (True, True)):
        e, off, rows, x, w, _, g = _layer(n, E, din, dout, pad, n + dout, form, order)
        dy = _wide(torch.randn(n, dout, device=DEV, generator=g).bfloat16(), pad)
        src, xin = x, x.double()
        if kept:
            src = im.Checkpoint(_out(n, din, pad, torch.int8), _out(n, -(-din // 32), pad, torch.uint8))
            im.checkpoint_store(x, src)
            xin = torch.from_numpy(_ckpt_ref(x)[2]).to(DEV)
        dxw = torch.zeros(n, din, device=DEV, dtype=torch.float64)
        dxs = torch.zeros_like(dxw)
        dww = torch.zeros(E, dout, din, device=DEV, dtype=torch.float64)
        dws, dbw = torch.zeros_like(dww), torch.zeros(E, dout, device=DEV, dtype=torch.float64)
        dbs, cnt = torch.zeros_like(dbw), torch.zeros(E, device=DEV, dtype=torch.float64)
        for k, r in enumerate(_by_expert(e, E)):
            d = dy[r].double()
            dxw[r], dxs[r] = d @ w[k].double(), d.abs() @ w[k].double().abs()
            dww[k], dws[k] = d.t() @ xin[r], d.abs().t() @ xin[r].abs()
            dbw[k], dbs[k], cnt[k] = d.sum(0), d.abs().sum(0), len(r)
        if relu:
            dxw[~(xin > 0)] = 0
        dx = _out(n, din, pad, torch.bfloat16)
        dx.fill_(5.0)
        dwf = _out(E * dout, din, pad, torch.float32)
        dwf.fill_(5.0)
        dw, db = dwf.unflatten(0, (E, dout)), torch.full((E, dout), 5.0, device=DEV)
        im.expert_linear_grad(dy, src, w, off, rows, dx, dw, db, relu_x=relu)
        _within(dx, dxw, 2 * dout * U * dxs + BF * dxw.abs(), "dx")
        _within(dw, dww, 2 * cnt[:, None, None] * U * dws, "dw")
        _within(db, dbw, 2 * cnt[:, None] * U * dbs, "db")
        _pad_kept(dx), _pad_kept(dwf)
        # each output alone, the same bits
        dx2, db2 = _out(n, din, pad, torch.bfloat16), torch.full((E, dout), 5.0, device=DEV)
        dw2 = _out(E * dout, din, pad, torch.float32).unflatten(0, (E, dout))
        im.expert_linear_grad(dy, src, w, off, rows, dx=dx2, relu_x=relu)
        im.expert_linear_grad(dy, src, w, off, rows, dw=dw2)
        im.expert_linear_grad(dy, None, w, off, rows, db=db2)
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)


def test_expert_linear_grad_long_groups():
    """Groups of several pieces of the weight gradient beside short and empty ones."""
    n, E, din, dout = 20000, 4, 96, 40
    g = _gen(8)
    e = torch.where(torch.rand(n, device=DEV, generator=g) < 0.9, 1, 3).to(torch.int32)
    e[5] = 0
    off, rows = torch.zeros(E + 1, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    im.group_rows(e, off, rows)
    x, dy = (torch.randn(n, d, device=DEV, generator=g).bfloat16() for d in (din, dout))
    w = torch.randn(E, dout, din, device=DEV, generator=g).bfloat16()
    dw, db = torch.full((E, dout, din), 5.0, device=DEV), torch.full((E, dout), 5.0, device=DEV)
    im.expert_linear_grad(dy, x, w, off, rows, dw=dw, db=db)
    for k, r in enumerate(_by_expert(e, E)):
        d, v = dy[r].double(), x[r].double()
        _within(dw[k], d.t() @ v, 2 * len(r) * U * (d.abs().t() @ v.abs()), "dw %d" % k)
        _within(db[k], d.sum(0), 2 * len(r) * U * d.abs().sum(0), "db %d" % k)
    assert not dw[2].any() and not db[2].any()
    dw2 = torch.zeros_like(dw)
    im.expert_linear_grad(dy, x, w, off, rows, dw=dw2)
    assert torch.equal(dw, dw2)


def test_expert_linear_grad_no_rows():
    E, din, dout = 3, 20, 10
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    x, dy = (torch.zeros(0, d, dtype=torch.bfloat16, device=DEV) for d in (din, dout))
    w = torch.zeros(E, dout, din, dtype=torch.bfloat16, device=DEV)
    dw, db = torch.full((E, dout, din), 5.0, device=DEV), torch.full((E, dout), 5.0, device=DEV)
    im.expert_linear_grad(dy, x, w, off, None, torch.zeros_like(x), dw, db)
    assert not dw.any() and not db.any()
    im.expert_linear(x, w, None, off, None, torch.zeros_like(dy))


def test_expert_layer_keeps_bad_rows_apart():
    """A row with NaN or infinity, and weights of another expert with them, touch no other row;
    a checkpoint's NaN block masks its rows' dx."""
    n, E, din, dout = 300, 3, 100, 70
    e, off, rows, x, w, b, g = _layer(n, E, din, dout, 4, 21)
    x[17, 3], x[40, 99] = float("nan"), float("inf")
    w[2, 5, 7] = float("nan")
    y = torch.zeros(n, dout, dtype=torch.bfloat16, device=DEV)
    im.expert_linear(x, w, b, off, rows, y)
    bad = ~torch.isfinite(y.float())
    expect = (e == 2)[:, None] & (torch.arange(dout, device=DEV) == 5)
    expect[17] = True
    expect[40] = True
    assert torch.equal(bad, expect)
    im.expert_linear(x, w, b, off, rows, y, relu=True)
    assert torch.isnan(y[17]).all()
    dy = torch.randn(n, dout, device=DEV, generator=g).bfloat16()
    ck = im.Checkpoint.empty(n, din)
    im.checkpoint_store(x, ck)
    dx = torch.zeros(n, din, dtype=torch.bfloat16, device=DEV)
    im.expert_linear_grad(dy, ck, w, off, rows, dx=dx, relu_x=True)
    assert not dx[17, :32].any() and not dx[40, 96:].any()
    dw = torch.zeros(E, dout, din, device=DEV)
    im.expert_linear_grad(dy, x, w, off, rows, dw=dw)
    for k in range(E):
        cols = set(torch.nonzero(~torch.isfinite(dw[k]).all(0)).flatten().tolist())
        assert cols == {c for r, c in ((17, 3), (40, 99)) if int(e[r]) == k}


def test_expert_layer_odd_index_arrays():
    """Entries of `rows` outside [0, n) are skipped, offsets are held within [0, n]."""
    n, E, din, dout = 200, 2, 40, 36
    e, off, rows, x, w, b, g = _layer(n, E, din, dout, 0, 5)
    ref = torch.zeros(n, dout, device=DEV)
    im.expert_linear(x, w, b, off, rows, ref)
    rows2 = rows.clone()
    rows2[3], rows2[150] = -1, 2 ** 31 - 1
    y = torch.full((n, dout), 7.0, device=DEV)
    im.expert_linear(x, w, b, off, rows2, y)
    skipped = [int(rows[3]), int(rows[150])]
    assert bool((y[skipped] == 7).all())
    keep = torch.ones(n, dtype=torch.bool, device=DEV)
    keep[skipped] = False
    assert torch.equal(y[keep], ref[keep])
    dy = torch.randn(n, dout, device=DEV, generator=g).bfloat16()
    dw, db = torch.zeros(E, dout, din, device=DEV), torch.zeros(E, dout, device=DEV)
    im.expert_linear_grad(dy, x, w, off, rows2, dw=dw, db=db)
    for k in range(E):
        r = torch.nonzero((e == k) & keep).flatten()
        d, v = dy[r].double(), x[r].double()
        _within(dw[k], d.t() @ v, 2 * n * U * (d.abs().t() @ v.abs()), "dw")
        _within(db[k], d.sum(0), 2 * n * U * d.abs().sum(0), "db")
    wild = torch.tensor([-5, int(off[1]), 2 ** 31 - 1], dtype=torch.int32, device=DEV)
    im.expert_linear(x, w, b, wild, rows, y)
    assert torch.equal(y, ref)


def test_expert_linear_grad_against_differences():
    """dx, dw and db against central differences of the float64 forward (a bilinear function:
    the differences are exact up to float64); dx adds one bf16 rounding a value."""
    n, E, din, dout = 40, 3, 31, 22
    e, off, rows, x, w, b, g = _layer(n, E, din, dout, 0, 77)
    dy = torch.randn(n, dout, device=DEV, generator=g).bfloat16()
    dx = torch.zeros(n, din, dtype=torch.bfloat16, device=DEV)
    dw, db = torch.zeros(E, dout, din, device=DEV), torch.zeros(E, dout, device=DEV)
    im.expert_linear_grad(dy, x, w, off, rows, dx, dw, db)

    def loss(x, w, b):
        return sum(((x[r] @ w[k].t() + b[k]) * dy[r].double()).sum() for k, r in enumerate(_by_expert(e, E)))

    args = [x.double(), w.double(), b.double()]
    for k, (grad, rel) in enumerate(((dx, BF), (dw, 2 * n * U), (db, 2 * n * U))):
        v = torch.randn(args[k].shape, device=DEV, generator=g, dtype=torch.float64)
        up, dn = list(args), list(args)
        up[k], dn[k] = args[k] + v, args[k] - v
        diff = float((loss(*up) - loss(*dn)) / 2)
        dot = float((grad.double() * v).sum())
        assert abs(diff - dot) <= rel * float((grad.double() * v).abs().sum()) + \
            2 * 64 * U * float(v.abs().sum()) * 8


def test_rows_past_two_gib():
    """Offsets beyond 2^31 elements: the last rows of a long matrix."""
    n, d = (1 << 21) + 70, 1024
    x = torch.zeros(n, d, dtype=torch.bfloat16, device=DEV)
    last = torch.randn(64, d, device=DEV, generator=_gen(2)).bfloat16()
    x[-64:] = last
    y = torch.zeros_like(x)
    m, r = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    ck = im.Checkpoint.empty(n, d)
    im.layer_norm(x, None, None, y, m, r, checkpoint=ck)
    y2 = torch.zeros_like(last)
    im.layer_norm(last, None, None, y2)
    assert torch.equal(y[-64:], y2) and not y[:-64].any()
    small = im.Checkpoint.empty(64, d)
    im.checkpoint_store(last, small)
    assert torch.equal(ck.q[-64:], small.q) and torch.equal(ck.scale[-64:], small.scale)
    dx, dx2 = torch.zeros_like(x), torch.zeros_like(last)
    im.layer_norm_grad(x, ck, None, m, r, dx)
    im.layer_norm_grad(last, small, None, m[-64:], r[-64:], dx2)
    assert torch.equal(dx[-64:], dx2)
    # one expert's rows are the last ones
    off = torch.tensor([0, 0, 64], dtype=torch.int32, device=DEV)
    rows = torch.cat([torch.arange(n - 64, n, device=DEV), torch.arange(0, n - 64, device=DEV)]).to(torch.int32)
    w = torch.randn(2, 512, d, device=DEV, generator=_gen(3)).bfloat16()
    o = torch.ones(n, 512, dtype=torch.bfloat16, device=DEV)
    im.expert_linear(x, w, None, off, rows, o)
    o2 = torch.zeros(64, 512, dtype=torch.bfloat16, device=DEV)
    im.expert_linear(last, w[1:], None, torch.tensor([0, 64], dtype=torch.int32, device=DEV), None, o2)
    _within(o[-64:], o2.double(), 2 * BF * o2.double().abs() + 1e-2, "y")
    assert not o[:-64].any()


def test_streams_and_graph():
    """A layer's calls on a stream of their own, and replayed from a graph on changing inputs."""
    n, E, d, o = 700, 4, 96, 72
    e, off, rows, x, w, b, g = _layer(n, E, d, o, 0, 31)
    gamma = torch.randn(d, device=DEV, generator=g)
    t = dict(xn=torch.zeros_like(x), m=torch.zeros(n, device=DEV), r=torch.zeros(n, device=DEV),
             y=torch.zeros(n, o, dtype=torch.bfloat16, device=DEV), dn=torch.zeros_like(x),
             dx=torch.zeros_like(x), dw=torch.zeros(E, o, d, device=DEV), db=torch.zeros(E, o, device=DEV),
             dg=torch.zeros(d, device=DEV), dbt=torch.zeros(d, device=DEV), off=off, rows=rows)
    ck = im.Checkpoint.empty(n, d)
    ws = [im.group_rows_workspace(n, E), im.expert_linear_grad_workspace(n, E, d, o),
          im.layer_norm_grad_workspace(n, d)]

    def calls(stream=None):
        im.group_rows(e, off, rows, ws[0], stream=stream)
        im.layer_norm(x, gamma, None, t["xn"], t["m"], t["r"], checkpoint=ck, stream=stream)
        im.expert_linear(t["xn"], w, b, off, rows, t["y"], relu=True, stream=stream)
        im.expert_linear_grad(t["y"], t["xn"], w, off, rows, t["dn"], t["dw"], t["db"], workspace=ws[1],
                              stream=stream)
        im.layer_norm_grad(t["dn"], ck, gamma, t["m"], t["r"], t["dx"], t["dg"], t["dbt"], ws[2],
                           stream=stream)

    calls()
    torch.cuda.synchronize()
    ref = {k: v.clone() for k, v in t.items()}
    side = torch.cuda.Stream()
    for v in t.values():
        v.zero_()
    torch.cuda.synchronize()
    calls(side)
    side.synchronize()
    for k, v in t.items():
        assert torch.equal(v, ref[k]), k
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for step in range(4):
        e.copy_(torch.randint(-1, E, (n,), device=DEV, dtype=torch.int32, generator=g))
        x.copy_(torch.randn(n, d, device=DEV, generator=g).bfloat16())
        calls()
        torch.cuda.synchronize()
        ref = {k: v.clone() for k, v in t.items()}
        for v in t.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in t.items():
            assert torch.equal(v, ref[k]), (step, k)


def test_binding_refuses_tensors_that_do_not_fit():
    n, d = 8, 64
    x = torch.zeros(n, d, device=DEV)
    with pytest.raises(ValueError, match="y must be"):
        im.layer_norm(x, None, None, torch.zeros(n, d + 1, device=DEV))
    with pytest.raises(ValueError, match="y must be"):
        im.layer_norm(x, None, None, x.bfloat16())
    with pytest.raises(ValueError, match="lie together"):
        im.layer_norm(torch.zeros(d, n, device=DEV).t(), None, None, x)
    with pytest.raises(ValueError, match="gamma"):
        im.layer_norm(x, torch.zeros(d, device=DEV).double(), None, x.clone())
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        im.layer_norm(x.half(), None, None, x.half())
    with pytest.raises(ValueError, match="current device"):
        im.layer_norm(x, None, None, torch.zeros(n, d))
    with pytest.raises(ValueError, match="scale"):
        im.checkpoint_store(x, im.Checkpoint(torch.zeros(n, d, dtype=torch.int8, device=DEV),
                                             torch.zeros(n, 1, dtype=torch.uint8, device=DEV)))
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    w = torch.zeros(2, 16, d, dtype=torch.bfloat16, device=DEV)
    xb, y = x.bfloat16(), torch.zeros(n, 16, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError, match="offsets"):
        im.expert_linear(xb, w, None, off[:2], None, y)
    with pytest.raises(ValueError, match="w must be"):
        im.expert_linear(x, w, None, off, None, y)
    with pytest.raises(ValueError, match="one stride"):
        im.expert_linear(xb, torch.zeros(2, 20, d, dtype=torch.bfloat16, device=DEV)[:, :16], None, off, None, y)
    with pytest.raises(im.ImError, match="bf16 only") as ei:
        im.expert_linear(x, w.float(), None, off, None, y)
    assert ei.value.status == im.IM_ERR_UNSUPPORTED
    with pytest.raises(im.ImError, match="workspace"):
        im.expert_linear_grad(y, xb, w, off, None, dw=torch.zeros(2, 16, d, device=DEV),
                              workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(im.ImError, match="no output"):
        im.expert_linear_grad(y, xb, w, off, None)
    with pytest.raises(ValueError, match="rows must be"):
        im.group_rows(off, off, torch.zeros(2, dtype=torch.int32, device=DEV))


# ------------------------------------------- sizes of the large tiles, both ways of loading
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("n,E,din,dout,pad,form", [
    (17000, 5, 264, 1000, 0, "holes"), (17000, 5, 1000, 264, 0, "even"), (16500, 3, 270, 1023, 2, "holes"),
    (16500, 3, 270, 1023, 1, "even"), (30000, 40, 257, 801, 0, "even"), (16400, 2, 512, 896, 0, "one"),
])
def test_large_tiles(n, E, din, dout, pad, form, kept):
    e, off, rows, x, w, b, g = _layer(n, E, din, dout, pad, n + dout, form)
    y = _out(n, dout, pad, torch.bfloat16)
    y.fill_(5.0)
    im.expert_linear(x, w, b, off, rows, y, relu=True)
    dy = _wide(torch.randn(n, dout, device=DEV, generator=g).bfloat16(), pad)
    src, xin = x, x.double()
    if kept:
        src = im.Checkpoint(_out(n, din, pad, torch.int8), _out(n, -(-din // 32), pad, torch.uint8))
        im.checkpoint_store(x, src)
        xin = torch.from_numpy(_ckpt_ref(x)[2]).to(DEV)
    dx = _out(n, din, pad, torch.bfloat16)
    dx.fill_(5.0)
    dw, db = torch.full((E, dout, din), 5.0, device=DEV), torch.full((E, dout), 5.0, device=DEV)
    im.expert_linear_grad(dy, src, w, off, rows, dx, dw, db, relu_x=True)
    none = torch.ones(n, dtype=torch.bool, device=DEV)
    for k, r in enumerate(_by_expert(e, E)):
        none[r] = False
        v, d, m, wk = x[r].double(), dy[r].double(), xin[r], w[k].double()
        want = (v @ wk.t() + b[k].double()).clamp(min=0)
        _within(y[r], want, 2 * (din + 1) * U * (v.abs() @ wk.abs().t() + b[k].double().abs()) + BF * want, "y")
        want = (d @ wk) * (m > 0)
        _within(dx[r], want, 2 * dout * U * (d.abs() @ wk.abs()) + BF * want.abs(), "dx")
        _within(dw[k], d.t() @ m, 2 * len(r) * U * (d.abs().t() @ m.abs()), "dw")
        _within(db[k], d.sum(0), 2 * len(r) * U * d.abs().sum(0), "db")
    assert not y[none].any() and not dx[none].any()
    _pad_kept(y), _pad_kept(dx)
    dw2, db2 = torch.zeros_like(dw), torch.zeros_like(db)
    im.expert_linear_grad(dy, src, w, off, rows, dw=dw2, db=db2)
    assert torch.equal(dw, dw2) and torch.equal(db, db2)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("n,E,din,dout,pad", [(5000, 3, 300, 1000, 4), (5000, 3, 1000, 300, 8),
                                              (4900, 6, 1016, 1022, 2), (3000, 12, 520, 330, 6)])
def test_middle_tiles(n, E, din, dout, pad, kept):
    """Sizes of the tiles between the smallest and the largest; dx in a launch of its own."""
    e, off, rows, x, w, b, g = _layer(n, E, din, dout, pad, n + dout, "holes")
    x = _wide(x.clamp(min=0).contiguous(), pad)
    wy = torch.zeros(n, -(-dout // 8) * 8, dtype=torch.bfloat16, device=DEV)
    dy = wy[:, :dout]
    dy.copy_(torch.randn(n, dout, device=DEV, generator=g))
    y = _out(n, dout, pad, torch.bfloat16)
    im.expert_linear(x, w, b, off, rows, y)
    src, xin = x, x.double()
    if kept:
        src = im.Checkpoint.empty(n, din)
        im.checkpoint_store(x, src)
        xin = torch.from_numpy(_ckpt_ref(x)[2]).to(DEV)
    dx, plain = _out(n, din, pad, torch.bfloat16), _out(n, din, pad, torch.bfloat16)
    im.expert_linear_grad(dy, src, w, off, rows, dx=dx, relu_x=True)
    im.expert_linear_grad(dy, None, w, off, rows, dx=plain)
    none = torch.ones(n, dtype=torch.bool, device=DEV)
    for k, r in enumerate(_by_expert(e, E)):
        none[r] = False
        v, d, wk = x[r].double(), dy[r].double(), w[k].double()
        want = v @ wk.t() + b[k].double()
        _within(y[r], want, 2 * (din + 1) * U * (v.abs() @ wk.abs().t() + b[k].double().abs()) + BF * want.abs(), "y")
        want, size = d @ wk, d.abs() @ wk.abs()
        _within(plain[r], want, 2 * dout * U * size + BF * want.abs(), "dx")
        assert torch.equal(dx[r], torch.where(xin[r] > 0, plain[r], torch.zeros_like(plain[r])))
    assert not y[none].any() and not dx[none].any()
    _pad_kept(y), _pad_kept(dx)


# Rows whose last 32-block has 1 to 7 values: a lane's last eight are of two blocks, here of
# very different scales.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,pad", [(7, 33, 0), (300, 65, 0), (129, 519, 1), (40, 1031, 0), (9, 4097, 3)])
def test_last_values_of_two_blocks(n, d, pad, dtype):
    x, gamma, beta, g = _norm_inputs(n, d, pad, dtype, n + 5 * d)
    seam = d // 32 * 32
    x[:, seam:] *= 2.0 ** -12
    x[1::2, seam:] *= 2.0 ** 24
    ck = im.Checkpoint(_out(n, d, pad, torch.int8), _out(n, -(-d // 32), pad, torch.uint8))
    ck2 = im.Checkpoint(_out(n, d, pad, torch.int8), _out(n, -(-d // 32), pad, torch.uint8))
    y = _out(n, d, pad, dtype)
    m, r = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    im.layer_norm(x, gamma, beta, y, m, r, eps=1e-2, checkpoint=ck)
    im.checkpoint_store(x, ck2)
    back = _ckpt_ref(x)[2]
    for c in (ck, ck2):
        _check_ckpt(x, c)
        v = _out(n, d, pad, torch.float32)
        im.checkpoint_load(c, v)
        assert np.array_equal(v.cpu().numpy().astype(np.float64), np.asarray(back, np.float64))
        _pad_kept(c.q), _pad_kept(c.scale), _pad_kept(v)
    dy = _wide(torch.randn(n, d, device=DEV, generator=g).to(dtype), pad)
    dx, dg, db = _out(n, d, pad, dtype), torch.zeros(d, device=DEV), torch.zeros(d, device=DEV)
    im.layer_norm_grad(dy, ck, gamma, m, r, dx, dg, db)
    want, dgam, dbet, size, sg, sb, _ = _ngrad_ref(dy, torch.from_numpy(back).to(DEV), gamma, m, r)
    _within(dx, want, 64 * U * size + (BF * want.abs() if dtype == torch.bfloat16 else 0) + 1e-300, "dx")
    _within(dg, dgam, 80 * U * sg + 1e-300, "dgamma")
    _within(db, dbet, 80 * U * sb + 1e-300, "dbeta")
    _pad_kept(dx)


# Several passes of a block over rows of 256, 512 and 1024 lanes.
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("n,d", [(5200, 1030), (2600, 2050), (1500, 4101)])
def test_layer_norm_grad_many_wide_rows(n, d, kept):
    test_layer_norm_grad(n, d, 0, torch.bfloat16, kept)
    test_layer_norm_grad(n, d, 1, torch.float32, kept)


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("n,E,din,dout,pad", [(300, 4, 64, 64, 0), (300, 4, 65, 40, 0), (40, 3, 6, 5, 0),
                                              (5000, 4, 128, 64, 0)])
def test_expert_linear_grad_pairs_of_outputs(n, E, din, dout, pad, kept):
    """Any two of dx, dw and db, with and without the mask, the same bits as all three; without
    dw and the mask x need not be given."""
    e, off, rows, x, w, _, g = _layer(n, E, din, dout, pad, n + 3, "holes")
    dy = _wide(torch.randn(n, dout, device=DEV, generator=g).bfloat16(), pad)
    src = x
    if kept:
        src = im.Checkpoint.empty(n, din)
        im.checkpoint_store(x, src)

    def call(xin, relu, names):
        o = dict(dx=torch.full((n, din), 5.0, dtype=torch.bfloat16, device=DEV),
                 dw=torch.full((E, dout, din), 5.0, device=DEV), db=torch.full((E, dout), 5.0, device=DEV))
        o = {k: o[k] for k in names}
        im.expert_linear_grad(dy, xin, w, off, rows, relu_x=relu, **o)
        return o

    for relu in (False, True):
        want = call(src, relu, ("dx", "dw", "db"))
        for names in (("dx", "db"), ("dx", "dw"), ("dw", "db")):
            for k, v in call(src, relu, names).items():
                assert torch.equal(v, want[k]), (relu, names, k)
        if not relu:
            for k, v in call(None, False, ("dx", "db")).items():
                assert torch.equal(v, want[k]), k


def test_scratch_memory_on_a_side_stream(monkeypatch):
    """Calls on a side stream without workspaces, beside work of the current one: their memory is
    allocated on the side stream, and the results are those of the current stream."""
    n, E, d, o = 20000, 5, 96, 72
    e, off, rows, x, w, b, g = _layer(n, E, d, o, 0, 41)
    dy = torch.randn(n, o, device=DEV, generator=g).bfloat16()
    m, r = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    im.layer_norm(x, None, None, torch.zeros_like(x), m, r)
    t = dict(off=torch.zeros_like(off), rows=torch.zeros_like(rows), dw=torch.zeros(E, o, d, device=DEV),
             db=torch.zeros(E, o, device=DEV), dg=torch.zeros(d, device=DEV), dbt=torch.zeros(d, device=DEV))

    def calls(stream=None):
        im.group_rows(e, t["off"], t["rows"], stream=stream)
        im.expert_linear_grad(dy, x, w, off, rows, dw=t["dw"], db=t["db"], stream=stream)
        im.layer_norm_grad(x, x, None, m, r, dgamma=t["dg"], dbeta=t["dbt"], stream=stream)

    calls()
    ref = {k: v.clone() for k, v in t.items()}
    for v in t.values():
        v.zero_()
    torch.cuda.synchronize()
    side, seen, space = torch.cuda.Stream(), [], im._space

    def noted(nbytes):
        seen.append(torch.cuda.current_stream())
        return space(nbytes)

    monkeypatch.setattr(im, "_space", noted)
    busy = torch.ones(1 << 24, device=DEV)
    for k in range(8):
        busy = busy * 1.5       # frees a temporary that the current stream still reads
        calls(side)
    torch.cuda.synchronize()
    assert len(seen) == 24 and all(s == side for s in seen)
    for k, v in t.items():
        assert torch.equal(v, ref[k]), k


# float32 outputs (a policy's head) and dx without a mask, on each size of tile
@pytest.mark.parametrize("n,E,din,dout,pad,form", [
    (17000, 5, 264, 1000, 0, "holes"), (16500, 3, 270, 1023, 1, "holes"),      # the largest, both ways of loading
    (5000, 3, 300, 1000, 4, "holes"), (3000, 12, 520, 330, 0, "even"),         # 128 x 128 and 128 x 64
])
def test_fp32_outputs_of_large_tiles(n, E, din, dout, pad, form):
    e, off, rows, x, w, b, g = _layer(n, E, din, dout, pad, n + dout, form)
    for relu, bias in ((False, b), (True, None)):
        y = _out(n, dout, 3, torch.float32)
        y.fill_(5.0)
        im.expert_linear(x, w, bias, off, rows, y, relu=relu)
        none = torch.ones(n, dtype=torch.bool, device=DEV)
        for k, r in enumerate(_by_expert(e, E)):
            none[r] = False
            v, wk = x[r].double(), w[k].double()
            want, size = v @ wk.t(), v.abs() @ wk.abs().t()
            if bias is not None:
                want, size = want + b[k].double(), size + b[k].double().abs()
            _within(y[r], want.clamp(min=0) if relu else want, 2 * (din + 1) * U * size, "y")
        assert not y[none].any()
        _pad_kept(y)


@pytest.mark.parametrize("n,E,din,dout,pad", [(17000, 5, 1000, 264, 0), (16500, 3, 1023, 270, 1)])
def test_unmasked_dx_of_large_tiles(n, E, din, dout, pad):
    e, off, rows, _, w, _, g = _layer(n, E, din, dout, pad, n + dout, "holes")
    dy = _wide(torch.randn(n, dout, device=DEV, generator=g).bfloat16(), pad)
    dx = _out(n, din, pad, torch.bfloat16)
    dx.fill_(5.0)
    im.expert_linear_grad(dy, None, w, off, rows, dx=dx)
    none = torch.ones(n, dtype=torch.bool, device=DEV)
    for k, r in enumerate(_by_expert(e, E)):
        none[r] = False
        d, wk = dy[r].double(), w[k].double()
        want = d @ wk
        _within(dx[r], want, 2 * dout * U * (d.abs() @ wk.abs()) + BF * want.abs(), "dx")
    assert not dx[none].any()
    _pad_kept(dx)


# More experts than a wavefront has lanes, their rows divided among teams of blocks: of 64 x 64
# tiles and of 256 x 256 ones, of aligned and of odd rows.
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("n,E,din,dout,pad", [
    (3000, 70, 64, 64, 0), (6000, 70, 64, 104, 0), (9000, 200, 41, 72, 0),
    (20000, 70, 264, 200, 0), (20000, 200, 137, 264, 2),
])
def test_weight_gradient_of_many_experts(n, E, din, dout, pad, kept):
    g = _gen(n + E)
    # uneven, with long and empty ones on both sides of number 64
    share = 0.1 + torch.rand(E, device=DEV, generator=g)
    share[torch.tensor([5, 62, 66, E - 3])] = 0.08 * E
    share[torch.tensor([0, 7, 63, 64, 65, E - 1])] = 0.0
    e = torch.multinomial(share, n, replacement=True, generator=g).to(torch.int32)
    e[::50] = -1
    off, rows = torch.zeros(E + 1, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    im.group_rows(e, off, rows)
    x = _wide(torch.randn(n, din, device=DEV, generator=g).bfloat16(), pad)
    dy = _wide(torch.randn(n, dout, device=DEV, generator=g).bfloat16(), pad)
    w = torch.zeros(E, dout, din, dtype=torch.bfloat16, device=DEV)
    src, xin = x, x.double()
    if kept:
        src = im.Checkpoint(_out(n, din, pad, torch.int8), _out(n, -(-din // 32), pad, torch.uint8))
        im.checkpoint_store(x, src)
        xin = torch.from_numpy(_ckpt_ref(x)[2]).to(DEV)
    dw, db = torch.full((E, dout, din), 5.0, device=DEV), torch.full((E, dout), 5.0, device=DEV)
    im.expert_linear_grad(dy, src, w, off, rows, dw=dw, db=db)
    for k, r in enumerate(_by_expert(e, E)):
        d, m = dy[r].double(), xin[r]
        _within(dw[k], d.t() @ m, 2 * len(r) * U * (d.abs().t() @ m.abs()), "dw %d" % k)
        _within(db[k], d.sum(0), 2 * len(r) * U * d.abs().sum(0), "db %d" % k)


def test_mask_of_a_checkpoint():
    """From a checkpoint the ReLU's mask is that of the restored values: it differs from the mask
    of the activations at positive ones of half a step or less, and nowhere else."""
    n, E, din, dout = 700, 3, 200, 72
    e, off, rows, x, w, b, g = _layer(n, E, din, dout, 0, 55)
    h = x.clamp(min=0)
    dy = torch.randn(n, dout, device=DEV, generator=g).bfloat16()
    ck = im.Checkpoint.empty(n, din)
    im.checkpoint_store(h, ck)
    dx, exact = (torch.zeros(n, din, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    im.expert_linear_grad(dy, h, w, off, rows, dx=exact, relu_x=True)
    im.expert_linear_grad(dy, ck, w, off, rows, dx=dx, relu_x=True)
    step = torch.exp2(ck.scale.double() - 133).repeat_interleave(32, dim=1)[:, :din]
    lost = (h > 0) & (h.double() <= step / 2)
    assert 0 < int(lost.sum()) < 0.02 * int((h > 0).sum())
    assert torch.equal(dx, torch.where(lost, torch.zeros_like(exact), exact))
