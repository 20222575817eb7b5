"""The blocks of a recurrent policy on the GPU: 8-bit matrices, root-mean-square norm, products
in 8 bits, gated scan and their gradients, against plain forms in 64 bits."""
import zlib

import numpy as np
import pytest

from tests import recurrent_oracle as O

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_09821_amd import binding as im  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(*key):
    g = torch.Generator()
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def _rows(x, pad):
    """x on the GPU as rows of a wider array whose other columns hold NaN."""
    wide = torch.full((*x.shape[:-1], x.shape[-1] + pad), float("nan"), dtype=x.dtype, device="cuda")
    wide[..., :x.shape[-1]] = x.cuda()
    return wide[..., :x.shape[-1]]


def _np(t):
    return t.detach().float().cpu().double().numpy()


def _bytes(q):
    return q.view(torch.uint8).cpu().numpy()


def _filled(n, d, rows=1, spare=1):
    """A Block8 of 0xA5 with `spare` rows behind its own."""
    b = im.Block8.empty(n + spare, d, 1)
    b.q.view(torch.uint8).fill_(0xA5)
    scale = torch.full((-(-n // rows) + spare, b.scale.shape[1]), 0xA5, dtype=torch.uint8, device="cuda")
    return im.Block8(b.q[:n], scale[:-(-n // rows)], d, rows), b.q[n:], scale[-(-n // rows):]


# ------------------------------------------------------------------- 8 bits
def _values(n, d, kind, dtype, g):
    x = torch.randn(n, d, generator=g)
    if kind == "wide":        # magnitudes over the whole range, also within a block
        x = x * torch.exp2(torch.randint(-140, 120, (n, d), generator=g).float())
        x[:, ::3] *= 0
    elif kind == "ties":      # halves of steps, largest magnitudes next to 448 2^e
        x = torch.randint(-64, 65, (n, d), generator=g).float() * 0.25
        x[::2, 0] = 448.0 * 2.0 ** -3
        x[1::2, -1] = 449.0 * 2.0 ** -3 if dtype == "f32" else 450.0 * 2.0 ** -3
    elif kind == "bad":
        x[0, 0] = float("nan")
        x[-1, -1] = float("inf")
        x[n // 2, d // 2] = -float("inf")
    elif kind == "zero":
        x = x * 0
    return x.to(DT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("n,d,kind,pad", [
    (1, 1, "normal", 0), (1, 128, "wide", 0), (2, 7, "ties", 1), (127, 129, "normal", 3),
    (128, 128, "ties", 0), (130, 361, "wide", 0), (300, 40, "bad", 5), (257, 512, "normal", 0),
    (3, 1000, "zero", 0)])
def test_block8_store_and_load(n, d, kind, pad, rows, dtype):
    x = _values(n, d, kind, dtype, _gen(n, d, kind))
    src = _rows(x, pad)
    v = _np(x)
    want, want_t = O.pack8(v, rows), O.pack8(np.ascontiguousarray(v.T), rows)
    for with_c, with_t in ((True, True), (True, False), (False, True)):
        c, qrest, srest = _filled(n, d, rows)
        t, tqrest, tsrest = _filled(d, n, rows)
        im.block8_store(src, c if with_c else None, t if with_t else None)
        for b, (q, s), on in ((c, want, with_c), (t, want_t, with_t)):
            if on:
                np.testing.assert_array_equal(b.scale.cpu().numpy(), s)
                np.testing.assert_array_equal(_bytes(b.q), q)
            else:
                assert (_bytes(b.q) == 0xA5).all()
        for r in (qrest.view(torch.uint8), srest, tqrest.view(torch.uint8), tsrest):
            assert (r == 0xA5).all()
        if with_c:
            for out in DT:
                back = _rows(torch.zeros(n, d, dtype=DT[out]), pad)
                im.block8_load(c, back)
                exact = O.unpack8(*want, d, rows)
                if out == "bf16":     # exact from scale 3 on
                    low = np.repeat(np.repeat(want[1] < 3, rows, 0)[:n], 128, 1)[:, :d]
                    exact = np.where(low, _np(back), exact)
                np.testing.assert_array_equal(_np(back), exact.astype(np.float32).astype(np.float64))


def test_block8_all_codes():
    """Every e4m3 value at every scale whose block it is the largest of, and back."""
    v = torch.tensor(O.E4M3, dtype=torch.float64)
    for s in (0, 1, 3, 120, 127, 246):      # 448 2^120 is no float32
        x = torch.zeros(127, 128)
        x[:, 0] = float(448 * 2.0 ** (s - 127))
        x[:, 1] = (v * 2.0 ** (s - 127)).float()
        x[:, 2] = -x[:, 1]
        b = im.Block8.empty(127, 128)
        im.block8_store(x.cuda(), b)
        assert (b.scale.cpu() == s).all()
        q = _bytes(b.q)
        np.testing.assert_array_equal(q[:, 1], np.arange(127))
        np.testing.assert_array_equal(q[:, 2] & 0x7F, np.arange(127))
        back = torch.zeros(127, 128, device="cuda")
        im.block8_load(b, back)
        assert torch.equal(back.cpu(), x)


# --------------------------------------------------------------------- norm
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad", [(1, 1, 0), (3, 5, 0), (33, 8, 1), (65, 30, 2), (17, 64, 0), (9, 100, 0),
                                     (7, 128, 3), (5, 361, 0), (4, 513, 0), (67, 1024, 8), (3, 2047, 0),
                                     (2, 8192, 0), (2, 8191, 1)])
@pytest.mark.parametrize("res", [False, True])
def test_rms_norm(n, d, pad, res, dtype):
    g = _gen(n, d, res)
    x, r = torch.randn(n, d, generator=g).to(DT[dtype]), (3 * torch.randn(n, d, generator=g)).to(DT[dtype])
    x[0] *= 1e-3                                   # a row where eps counts
    if res:
        r[0] *= 1e-3
    gamma = 1 + 0.3 * torch.randn(d, generator=g)
    eps = 1e-6
    h64, rstd64, y64 = O.rms_norm(_np(x), _np(r) if res else None, gamma.double().numpy(), eps)
    xs, rs = _rows(x, pad), _rows(r, pad) if res else None
    y, h = _rows(torch.zeros_like(x), pad), _rows(torch.zeros_like(x), pad)
    rstd = torch.zeros(n, device="cuda")
    y8, qrest, srest = _filled(n, d)
    im.rms_norm(xs, gamma.cuda(), y, rstd, eps, rs, h, y8)
    # the sum of squares: 8 products a lane and log2(1024) sums, each off by a rounding; half of
    # that in its root, then a root, a quotient and two products
    k = 24 * O.U32
    cancel = 2 * O.U32 * (np.abs(_np(x)) + np.abs(_np(r))) if res else 0.0     # the sum's own rounding
    hmag = np.abs(h64) + cancel
    kr = k + (np.abs(cancel) * np.abs(h64)).sum(1) / np.maximum((h64 * h64).sum(1), 1e-30) if res else k
    assert (np.abs(_np(rstd) - rstd64) <= kr * rstd64).all()
    assert (np.abs(_np(h) - h64) <= O.HALF[dtype] * hmag * 1.01 + cancel).all()
    ytol = (np.reshape(kr, (-1, 1)) + 3 * O.U32) * np.abs(y64) + \
        cancel * rstd64[:, None] * np.abs(gamma.double().numpy())
    assert (np.abs(_np(y) - y64) <= ytol + O.HALF[dtype] * 1.01 * np.abs(y64)).all()
    # 8 bits: half a step of the value, or of the least step of its block
    back = torch.zeros(n, d, device="cuda")
    im.block8_load(y8, back)
    step = np.repeat(2.0 ** (y8.scale.cpu().numpy().astype(float) - 127), 128, 1)[:, :d]
    assert (np.abs(_np(back) - y64) <= 2.0 ** -4 * np.abs(y64) * 1.001 + 2.0 ** -10 * step + 2 * ytol).all()
    assert (_bytes(y8.q)[:, d:] == 0).all()
    assert (qrest.view(torch.uint8) == 0xA5).all() and (srest == 0xA5).all()
    if dtype == "f32":       # the same values as stored from y
        again = im.Block8.empty(n, d)
        im.block8_store(y, again)
        np.testing.assert_array_equal(_bytes(again.q), _bytes(y8.q))
        assert torch.equal(again.scale, y8.scale)
    # in place: h over the residual (or x), y over x
    if res:
        im.rms_norm(xs, gamma.cuda(), xs, None, eps, rs, rs)
        assert torch.equal(rs, h)
    else:
        im.rms_norm(xs, gamma.cuda(), xs, None, eps)
    assert torch.equal(xs, y)


def test_rms_norm_of_rows_that_are_not_finite():
    x = torch.randn(5, 200, generator=_gen(1))
    x[1, 3], x[2, 4], x[3] = float("nan"), float("inf"), 0.0
    y, rstd = torch.zeros(5, 200, device="cuda"), torch.zeros(5, device="cuda")
    y8 = im.Block8.empty(5, 200)
    im.rms_norm(x.cuda(), None, y, rstd, 1e-6, y8=y8)
    assert torch.isfinite(y[[0, 3, 4]]).all() and (y[3] == 0).all()
    assert torch.isnan(y[1]).all() and torch.isnan(rstd[1])
    assert rstd[2] == 0 and torch.isnan(y[2, 4]) and (y[2, :4] == 0).all()
    s = y8.scale.cpu()
    assert (s[1] == 255).all() and s[2, 0] == 255 and s[2, 1] == 0 and (s[3] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad", [(1, 1, 0), (3, 5, 0), (300, 8, 1), (65, 30, 2), (17, 64, 0), (9, 100, 0),
                                     (700, 128, 3), (41, 361, 0), (20, 513, 0), (67, 1024, 8), (40, 2047, 0),
                                     (33, 8192, 0)])
@pytest.mark.parametrize("res", [False, True])
def test_rms_norm_grad(n, d, pad, res, dtype):
    g = _gen(n, d, res, 2)
    h, dy, dh = (torch.randn(n, d, generator=g).to(DT[dtype]) for _ in range(3))
    gamma = 1 + 0.3 * torch.randn(d, generator=g)
    rstd = (1 / torch.sqrt(h.double().square().mean(1) + 1e-6)).float()
    dx64, dg64 = O.rms_norm_grad(_np(dy), _np(h), _np(dh) if res else None, gamma.double().numpy(),
                                 rstd.double().numpy())
    args = _rows(dy, pad), _rows(h, pad), gamma.cuda(), rstd.cuda()
    dx, dgamma = _rows(torch.zeros_like(h), pad), torch.full((d,), 9.0, device="cuda")
    dhs = _rows(dh, pad) if res else None
    im.rms_norm_grad(*args, dx, dgamma, dhs)
    # dx: the row's sum, 8 + 10 roundings of its terms' magnitudes; then few products
    u, gg = _np(h) * rstd.double().numpy()[:, None], _np(dy) * gamma.double().numpy()
    mag = rstd.double().numpy()[:, None] * (np.abs(gg) + np.abs(u) * np.abs(gg * u).mean(1, keepdims=True))
    mag = mag + (np.abs(_np(dh)) if res else 0)
    assert (np.abs(_np(dx) - dx64) <= 28 * O.U32 * mag + O.HALF[dtype] * 1.01 * np.abs(dx64)).all()
    # dgamma: a column's terms one after the other in fp32, at most all of them
    assert (np.abs(_np(dgamma) - dg64) <= (n + 8) * O.U32 * np.abs(_np(dy) * u).sum(0)).all()
    # each output alone, the same bits; in place
    only = torch.zeros(d, device="cuda")
    im.rms_norm_grad(*args, None, only, dhs)
    assert torch.equal(only, dgamma)
    for where in ([dhs] if res else []) + [args[0]]:
        im.rms_norm_grad(*args, where, None, dhs)
        assert torch.equal(where, dx)
        break
    im.rms_norm_grad(args[0][:0], args[1][:0], args[2], args[3][:0], None, only)
    assert (only == 0).all()


# ------------------------------------------------------------------ products
def _pair(x, rows, **k):
    b = im.Block8.empty(*x.shape, rows)
    im.block8_store(x.cuda(), b, **k)
    return b, O.unpack8(_bytes(b.q), b.scale.cpu().numpy(), x.shape[1], rows)


SIZES = [(1, 1, 1), (1, 361, 1024), (3, 128, 5), (33, 129, 69), (64, 512, 130), (128, 256, 128), (129, 640, 127),
         (300, 77, 260), (513, 1024, 384), (1000, 1100, 200), (31, 2500, 33),
         (16384, 40, 300), (17001, 1100, 69)]


@pytest.mark.parametrize("n,i,o", SIZES)
@pytest.mark.parametrize("rows", [(1, 128), (1, 1), (128, 1)])
@pytest.mark.parametrize("out", ["f32", "bf16", "8", "both", "both32"])
def test_linear8(n, i, o, rows, out):
    g = _gen(n, i, o)
    # blocks of their own scale
    x = torch.randn(n, i, generator=g) * torch.exp2(torch.randint(-8, 9, (n, i // 128 + 1), generator=g).float()
                                                    ).repeat_interleave(128, 1)[:, :i]
    w = torch.randn(o, i, generator=g) * torch.exp2(torch.randint(-4, 5, (o, 1), generator=g).float()) * i ** -0.5
    bias = torch.randn(o, generator=g) if (n + o) % 2 else None
    relu = out in ("bf16", "both")
    x8, xv = _pair(x, rows[0])
    w8, wv = _pair(w, rows[1])
    y64 = xv @ wv.T + (0 if bias is None else bias.double().numpy())
    # products are exact; sums of i and the bias in any order, each off by a step at most
    mass = np.abs(xv) @ np.abs(wv).T
    tol = (i + 2) * 2 * O.U32 * (mass + (0 if bias is None else np.abs(bias.double().numpy())))
    if out == "bf16":
        # 8-bit MFMA adds eight products to a unit of 2^-13 of the power of two of the largest:
        # the seven others lose less than a unit each, 7 2^-13 of the largest's magnitude at most
        tol = tol + 7 * 2.0 ** -13 * mass
    if relu:
        y64 = np.maximum(y64, 0)
    behind = None
    if out == "8":
        y = None
    else:
        y = _rows(torch.full((n + 1, o), 7.0, dtype=DT["f32" if out in ("f32", "both32") else "bf16"]), n % 3)
        y, behind = y[:n], y[n:]
    y8, qrest, srest = _filled(n, o) if out in ("8", "both", "both32") else (None, None, None)
    im.linear8(x8, w8, None if bias is None else bias.cuda(), y, y8=y8, relu=relu)
    if y is not None:
        half = O.HALF["f32" if out in ("f32", "both32") else "bf16"]
        assert (np.abs(_np(y) - y64) <= tol + half * 1.01 * (np.abs(y64) + tol)).all()
        assert (behind == 7).all()
    if y8 is not None:
        back = torch.zeros(n, o, device="cuda")
        im.block8_load(y8, back)
        step = np.repeat(2.0 ** (y8.scale.cpu().numpy().astype(float) - 127), 128, 1)[:, :o]
        assert (np.abs(_np(back) - y64) <= 2.0 ** -4 * 1.001 * (np.abs(y64) + tol) + 2.0 ** -10 * step + tol).all()
        assert (_bytes(y8.q)[:, o:] == 0).all()
        assert (qrest.view(torch.uint8) == 0xA5).all() and (srest == 0xA5).all()


@pytest.mark.parametrize("n,i,o", [(5, 300, 40), (200, 300, 150), (700, 130, 129)])
def test_linear8_of_whole_numbers_is_exact(n, i, o):
    """Whole numbers that e4m3 holds, their sums below 2^24: every product and sum is exact."""
    g = _gen(n, i, o, 7)
    x, w = torch.randint(-15, 16, (n, i), generator=g).float(), torch.randint(-15, 16, (o, i), generator=g).float()
    x8, w8 = _pair(x, 1)[0], _pair(w, 128)[0]
    y = torch.zeros(n, o, device="cuda")
    y8 = im.Block8.empty(n, o)
    im.linear8(x8, w8, None, y, y8=y8)
    assert torch.equal(y.cpu(), x @ w.t())
    again = im.Block8.empty(n, o)
    im.block8_store(y, again)
    assert torch.equal(again.q.view(torch.uint8), y8.q.view(torch.uint8)) and torch.equal(again.scale, y8.scale)


def test_linear8_of_many_rows():
    """The largest tiles, with ends in both directions, every output."""
    n, i, o = 66000, 200, 300
    g = _gen(n)
    x8, w8 = im.Block8.empty(n, i), im.Block8.empty(o, i, 128)
    x = torch.randn(n, i, generator=g).cuda()
    im.block8_store(x, x8)
    im.block8_store(torch.randn(o, i, generator=g).cuda(), w8)
    bias = torch.randn(o, generator=g).cuda()
    xv, wv = (torch.zeros(*b.shape, device="cuda") for b in (x8, w8))
    im.block8_load(x8, xv)
    im.block8_load(w8, wv)
    want = (xv.double() @ wv.double().t() + bias.double()).clamp(min=0)
    mass = xv.double().abs() @ wv.double().abs().t() + bias.double().abs()
    for out in ("f32", "bf16", "8"):
        y8 = im.Block8.empty(n, o) if out != "bf16" else None
        y = torch.full((n + 1, o), 7.0, device="cuda", dtype=DT["bf16" if out == "bf16" else "f32"])
        im.linear8(x8, w8, bias, None if out == "8" else y[:n], y8=y8, relu=True)
        tol = (i + 2) * 2 * O.U32 * mass + (7 * 2.0 ** -13 * mass if out == "bf16" else 0)
        if out != "8":
            half = O.HALF["f32" if out == "f32" else "bf16"] * 1.01
            assert bool(((y[:n].double() - want).abs() <= tol + half * (want + tol)).all())
            assert (y[n] == 7).all()
        if y8 is not None:
            im.block8_load(y8, y[:n])
            step = torch.exp2(y8.scale.double() - 127).repeat_interleave(128, 1)[:, :o]
            assert bool(((y[:n].double() - want).abs() <= 2.0 ** -4 * 1.001 * (want + tol) + 2.0 ** -10 * step + tol).all())
            assert not y8.q.view(torch.uint8)[:, o:].any()


@pytest.mark.parametrize("i,o,rows,pad", [(40, 69, (1, 128), 1), (129, 100, (128, 1), 0), (300, 801, (1, 1), 3), (512, 1024, (1, 128), 0),
                                          (640, 897, (128, 128), 8), (1000, 1100, (1, 128), 2)])
def test_linear8_of_panels(i, o, rows, pad):
    """Many rows to bf16: one to eight blocks of k, ends in both directions, a row that is NaN and one of zeros."""
    n = 65601
    g = _gen(i, o)
    x = torch.randn(n, i, generator=g)
    x[7 if rows[0] == 1 else slice(0, 128)] = 0.0
    x[n - 1, i - 1] = float("nan")
    x8, w8 = im.Block8.empty(n, i, rows[0]), im.Block8.empty(o, i, rows[1])
    im.block8_store(x.cuda(), x8)
    im.block8_store(torch.randn(o, i, generator=g).cuda(), w8)
    bias = torch.randn(o, generator=g).cuda()
    xv, wv = (torch.zeros(*b.shape, device="cuda") for b in (x8, w8))
    im.block8_load(x8, xv)
    im.block8_load(w8, wv)
    bad = torch.isnan(xv).any(1)
    assert 1 <= int(bad.sum()) <= rows[0]
    xv[bad] = 0.0
    want = (xv.double() @ wv.double().t() + bias.double()).clamp(min=0)
    mass = xv.double().abs() @ wv.double().abs().t() + bias.double().abs()
    y = _rows(torch.full((n + 1, o), 7.0, dtype=torch.bfloat16), pad)
    im.linear8(x8, w8, bias, y[:n], relu=True)
    assert torch.isnan(y[:n][bad]).all() and (y[n] == 7).all() and torch.isnan(y._base[:, o:]).all()
    # as for the tiles: eight products are added to a unit of 2^-13 of the largest's power of two
    tol = (i + 2) * 2 * O.U32 * mass + 7 * 2.0 ** -13 * mass
    err = (y[:n].double() - want).abs()
    assert bool((err <= tol + O.HALF["bf16"] * 1.01 * (want + tol))[~bad].all())


@pytest.mark.parametrize("n", [3, 40, 200, 600, 66000])
def test_linear8_of_blocks_that_are_not_finite(n):
    """A row with a NaN or an infinity is NaN in y, and no other; the extreme scales."""
    g = _gen(n, 8)
    x, w = torch.randn(n, 300, generator=g), torch.randn(200, 300, generator=g)
    x[1, 5], x[2, 299] = float("nan"), float("inf")
    x[0] = 0.0
    x8, w8 = _pair(x, 1)[0], _pair(w, 1)[0]
    y = torch.zeros(n, 200, device="cuda")
    im.linear8(x8, w8, None, y, relu=True)
    bad = torch.isnan(y).all(1).cpu()
    assert bad[1] and bad[2] and not torch.isnan(y[~bad.cuda()]).any() and int(bad.sum()) == 2
    assert (y[0] == 0).all()
    yb, y8 = torch.zeros(n, 200, device="cuda", dtype=torch.bfloat16), im.Block8.empty(n, 200)
    im.linear8(x8, w8, None, yb, relu=True)
    im.linear8(x8, w8, None, None, y8=y8, relu=True)
    im.block8_load(y8, y)
    for t in (yb, y):
        assert torch.equal(torch.isnan(t).all(1).cpu(), bad) and torch.equal(torch.isnan(t).any(1).cpu(), bad)
    big, small = torch.full((n, 128), 3.0e38), torch.full((4, 128), 1e-36)
    b8, bv = _pair(big, 1)
    s8, sv = _pair(small, 1)
    y = torch.zeros(n, 4, device="cuda")
    im.linear8(b8, s8, None, y)
    np.testing.assert_allclose(_np(y), bv @ sv.T, rtol=130 * 2 * O.U32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,i,o,relu,pad", [
    (1, 1, 1, False, 0), (1, 361, 64, True, 0), (5, 40, 200, True, 3), (128, 128, 128, False, 0),
    (130, 361, 129, True, 1), (1000, 257, 96, False, 0), (4097, 69, 300, True, 0), (9000, 130, 20, False, 5),
    (4095, 361, 300, True, 1), (1024, 1000, 1020, False, 0), (6500, 640, 1000, True, 2)])
def test_linear8_grad(n, i, o, relu, pad, dtype):
    g = _gen(n, i, o, 3)
    x, w = torch.randn(n, i, generator=g), torch.randn(o, i, generator=g)
    dy = (torch.randn(n, o, generator=g) * 1e-3).to(DT[dtype])
    y = torch.randn(n, o, generator=g).clamp(min=0).to(DT[dtype])
    xt, wt = im.Block8.empty(i, n), im.Block8.empty(i, o, 128)
    im.block8_store(x.cuda(), None, xt)
    im.block8_store(w.cuda(), None, wt)
    xv = O.unpack8(_bytes(xt.q), xt.scale.cpu().numpy(), n).T
    wv = O.unpack8(_bytes(wt.q), wt.scale.cpu().numpy(), o, 128).T
    m = _np(dy) * ((_np(y) > 0) if relu else 1)
    rowwise = O.unpack8(*O.pack8(m), o)
    colwise = O.unpack8(*O.pack8(np.ascontiguousarray(m.T)), n).T
    dys, ys = _rows(dy, pad), _rows(y, pad) if relu else None
    dx, dw = _rows(torch.zeros(n, i, dtype=DT[dtype]), pad), _rows(torch.zeros(o, i), pad)
    db = torch.zeros(o, device="cuda")
    im.linear8_grad(dys, xt, wt, dx, dw, db, y=ys)
    dx64, dw64, db64 = rowwise @ wv, colwise.T @ xv, m.sum(0)
    tol = ((o + 2) * 2 * O.U32 + (7 * 2.0 ** -13 if dtype == "bf16" else 0)) * (np.abs(rowwise) @ np.abs(wv))
    assert (np.abs(_np(dx) - dx64) <= tol + O.HALF[dtype] * 1.01 * (np.abs(dx64) + tol)).all()
    assert (np.abs(_np(dw) - dw64) <= (n + 2) * 2 * O.U32 * (np.abs(colwise).T @ np.abs(xv))).all()
    assert (np.abs(_np(db) - db64) <= (128 + 2) * O.U32 * np.abs(m).sum(0)).all()
    # each alone: the same bits
    for k in range(3):
        outs = [torch.full_like(t, 7.0) if j == k else None for j, t in enumerate((dx, dw, db))]
        im.linear8_grad(dys, xt if k == 1 else None, wt if k == 0 else None, *outs, y=ys)
        assert torch.equal(outs[k], (dx, dw, db)[k])


def test_linear8_grad_of_no_rows():
    dw, db = torch.ones(40, 24, device="cuda"), torch.ones(40, device="cuda")
    dx = torch.zeros(0, 24, dtype=torch.bfloat16, device="cuda")
    wt = im.Block8.empty(24, 40, 128)
    xt = im.Block8(torch.zeros(24, 0, dtype=torch.float8_e4m3fn, device="cuda"),
                   torch.zeros(24, 0, dtype=torch.uint8, device="cuda"), 0)
    im.linear8_grad(torch.zeros(0, 40, dtype=torch.bfloat16, device="cuda"), xt, wt, dx, dw, db)
    assert (dw == 0).all() and (db == 0).all()


# ----------------------------------------------------------------------- scan
def _scan_case(T, n, d, dtype, done, state, key):
    g = _gen(T, n, d, key)
    gate = (2 + 2 * torch.randn(T, n, d, generator=g)).to(DT[dtype])
    x, dh = torch.randn(T, n, d, generator=g).to(DT[dtype]), torch.randn(T, n, d, generator=g).to(DT[dtype])
    flags = torch.zeros(2, T, n, dtype=torch.uint8)
    if done:
        flags = (torch.rand(2, T, n, generator=g) < 0.1).to(torch.uint8) * 3
    c0 = torch.randn(n, d, generator=g) if state else torch.zeros(n, d)
    dc = torch.randn(n, d, generator=g) if state else torch.zeros(n, d)
    return gate, x, dh, flags, c0, dc


def _lay(x, how):
    """x [T][n][d] on the GPU: dense, as padded rows, as halves of wider rows, or env by env."""
    if how == "dense":
        return x.cuda().contiguous()
    if how == "padded":
        return _rows(x, 3)
    if how == "halves":
        return _rows(x, x.shape[-1])
    t = torch.full((x.shape[1], x.shape[0], x.shape[2] + 1), float("nan"), dtype=x.dtype, device="cuda")
    t[..., :-1] = x.transpose(0, 1).cuda()
    return t[..., :-1].transpose(0, 1)


SCANS = [(1, 1, 1), (1, 64, 512), (2, 3, 7), (15, 5, 33), (16, 2, 8), (17, 9, 130), (32, 40, 64), (33, 1, 361),
         (100, 3, 20), (64, 2000, 12), (1000, 2, 37), (4099, 1, 6), (700, 150, 16)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,n,d", SCANS)
@pytest.mark.parametrize("done,state,how", [(True, True, "dense"), (False, False, "padded"), (True, False, "halves"),
                                            (True, True, "by env")])
def test_gated_scan_and_its_gradient(T, n, d, done, state, how, dtype):
    gate, x, dh, flags, c0, dc = _scan_case(T, n, d, dtype, done, state, 1)
    end = (flags[0] | flags[1]).numpy() != 0
    h64, before, last, eh, ebefore, elast = O.scan(_np(gate), _np(x), end, _np(c0))
    gs, xs, dhs = _lay(gate, how), _lay(x, how), _lay(dh, how)
    h = _lay(torch.zeros_like(x), how)
    f = _rows(flags, 2) if False else flags.cuda()
    term, trunc = (f[0], f[1]) if done else (None, None)
    K = -(-T // 16)
    keep = torch.full((K + 1, n, d), 7.0, device="cuda")
    s0 = c0.cuda() if state else None
    out = torch.zeros(n, d, device="cuda")
    im.gated_scan(gs, xs, h, s0, out, keep[:K], term, trunc)
    half = O.HALF[dtype]
    assert (np.abs(_np(h) - h64) <= eh + half * 1.01 * (np.abs(h64) + eh)).all()
    assert (np.abs(_np(out) - last) <= elast).all()
    assert (np.abs(_np(keep[:K]) - before[::16]) <= ebefore[::16]).all()
    assert (keep[K] == 7).all()
    if how != "dense":
        base = h._base if h._base is not None else h
        assert int(torch.isnan(base).sum()) == base.numel() - h.numel()
    # state in place
    if state:
        again = c0.cuda()
        h2 = _lay(torch.zeros_like(x), how)
        im.gated_scan(gs, xs, h2, again, again, None, term, trunc)
        assert torch.equal(again, out) and torch.equal(h2, h)
    # the gradient
    dgate64, dx64, dst64, eg, ex, es = O.scan_grad(_np(dh), _np(gate), _np(x), end, before, ebefore, _np(dc))
    dgate, dx = _lay(torch.zeros_like(x), how), _lay(torch.zeros_like(x), how)
    dst = torch.zeros(n, d, device="cuda")
    ds = dc.cuda() if state else None
    im.gated_scan_grad(dhs, gs, xs, keep[:K], dgate, dx, ds, dst, term, trunc)
    assert (np.abs(_np(dgate) - dgate64) <= eg + half * 1.01 * (np.abs(dgate64) + eg)).all()
    assert (np.abs(_np(dx) - dx64) <= ex + half * 1.01 * (np.abs(dx64) + ex)).all()
    assert (np.abs(_np(dst) - dst64) <= es).all()
    if state:
        im.gated_scan_grad(dhs, gs, xs, keep[:K], dgate, dx, ds, ds, term, trunc)
        assert torch.equal(ds, dst)


@pytest.mark.parametrize("T", [40, 600])
def test_gated_scan_of_extreme_gates(T):
    """Gates of plus and minus infinity keep and replace the state exactly; a NaN stays in its
    env and channel, up to the episode's end."""
    n, d = 3, 8
    gate, x = torch.zeros(T, n, d), torch.randn(T, n, d, generator=_gen(T))
    gate[:, 0], gate[:, 1] = float("inf"), -float("inf")
    gate[:, 2] = torch.tensor([1e4, -1e4, 89.0, -89.0, 104.0, -104.0, 0.0, 3e38])
    state = torch.randn(n, d, generator=_gen(T, 1))
    x[5, 2, 6] = float("nan")
    flags = torch.zeros(T, n, dtype=torch.uint8)
    flags[T // 2, 2] = 1
    h, keep = torch.zeros(T, n, d, device="cuda"), torch.zeros(-(-T // 16), n, d, device="cuda")
    out = torch.zeros(n, d, device="cuda")
    im.gated_scan(gate.cuda(), x.cuda(), h, state.cuda(), out, keep, flags.cuda())
    h = h.cpu()
    assert torch.equal(h[:, 0], state[0].expand(T, d)) and torch.equal(h[:, 1], x[:, 1])
    assert torch.isnan(h[5:T // 2 + 1, 2, 6]).all() and int(torch.isnan(h).sum()) == T // 2 - 4
    dgate, dx = torch.zeros(T, n, d, device="cuda"), torch.zeros(T, n, d, device="cuda")
    im.gated_scan_grad(torch.ones(T, n, d, device="cuda"), gate.cuda(), x.cuda(), keep, dgate, dx,
                       terminated=flags.cuda())
    dgate, dx = dgate.cpu(), dx.cpu()
    assert (dgate[:, :2] == 0).all() and (dx[:, 0] == 0).all() and (dx[:, 1] == 1).all()
    assert not torch.isnan(dx).any() and torch.isnan(dgate[5:T // 2 + 1, 2, 6]).all()
    assert int(torch.isnan(dgate).sum()) == T // 2 - 4


def test_gated_scan_of_no_steps():
    a = torch.zeros(0, 3, 5, device="cuda")
    state, out = torch.randn(3, 5, device="cuda"), torch.zeros(3, 5, device="cuda")
    im.gated_scan(a, a, a, state, out)
    assert torch.equal(out, state)
    out.zero_()
    im.gated_scan_grad(a, a, a, a, a, a, state, out)
    assert torch.equal(out, state)


def test_gated_scan_step_by_step():
    """A rollout's steps one at a time give the bits of one call over all of them."""
    T, n, d = 20, 6, 24
    gate, x, _, flags, c0, _ = _scan_case(T, n, d, "f32", True, True, 5)
    gate, x, f = gate.cuda(), x.cuda(), flags.cuda()
    whole, one = torch.zeros(T, n, d, device="cuda"), torch.zeros(T, n, d, device="cuda")
    s1, s2 = c0.cuda(), c0.cuda()
    im.gated_scan(gate, x, whole, s1, s1, None, f[0], f[1])
    for t in range(T):
        im.gated_scan(gate[t:t + 1], x[t:t + 1], one[t:t + 1], s2, s2, None, f[0, t:t + 1], f[1, t:t + 1])
    assert torch.equal(one, whole) and torch.equal(s1, s2)


@pytest.mark.parametrize("T", [20, 3000])
def test_gated_scan_of_other_layouts(T):
    """Flags that are bool, or one of the two; gates that all envs share; strides of both orders."""
    n, d = 5, 40
    gate, x, dh, flags, c0, _ = _scan_case(T, n, d, "bf16", True, True, 6)
    gate[:] = gate[:, :1]
    g, xs, f = gate.cuda(), x.cuda(), flags.cuda()
    either = f[0] | f[1]
    want, h = torch.zeros_like(xs), torch.zeros_like(xs)
    im.gated_scan(g, xs, want, c0.cuda(), None, None, f[0], f[1])
    shared = g[:, :1].expand(T, n, d)
    for term, trunc in ((either, None), (None, either != 0), (f[0] != 0, f[1] != 0)):
        h.zero_()
        im.gated_scan(shared, xs, h, c0.cuda(), None, None, term, trunc)
        assert torch.equal(h, want)
    wide = torch.zeros(T, n + 3, dtype=torch.uint8, device="cuda")
    wide[:, :n] = either
    by_env = xs.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.zeros(n, T, d, dtype=x.dtype, device="cuda").transpose(0, 1)
    im.gated_scan(g, by_env, out, c0.cuda(), None, None, wide[:, :n])
    assert torch.equal(out, want)


# --------------------------------------------------------------- far offsets
def test_gated_scan_of_envs_far_apart():
    """Rows of one step 36 MB apart, env by env, give the bits of rows that lie together."""
    T, n, d = 70000, 3, 256
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    gate, x = (torch.randn(T, n, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    far = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (gate, x)]
    want, h = torch.zeros_like(x), torch.zeros_like(far[1])
    keep, keep2 = (torch.zeros(-(-T // 16), n, d, device="cuda") for _ in range(2))
    im.gated_scan(gate, x, want, keep=keep)
    im.gated_scan(*far, h, keep=keep2)
    assert torch.equal(h, want) and torch.equal(keep, keep2)
    outs = [torch.zeros_like(x) for _ in range(2)] + [torch.zeros_like(far[1]) for _ in range(2)]
    im.gated_scan_grad(x, gate, x, keep, *outs[:2])
    im.gated_scan_grad(far[1], *far, keep, *outs[2:])
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


def test_offsets_that_pass_32_bits():
    """Arrays of more than 4 GB: their last rows as alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    n, d = 2200064, 1024
    x = torch.randint(-15, 16, (n, d), device="cuda", generator=g, dtype=torch.int8).bfloat16()
    y, h = torch.empty_like(x), torch.empty_like(x)
    rstd = torch.zeros(n, device="cuda")
    x8, xt = im.Block8.empty(n, d), im.Block8.empty(d, n)
    im.rms_norm(x, None, y, rstd, residual=x, h=h, y8=x8)
    tail = slice(n - 128, n)
    xl, yl, rl, l8, lt = (x[tail].contiguous(), torch.zeros(128, d, dtype=x.dtype, device="cuda"),
                          torch.zeros(128, device="cuda"), im.Block8.empty(128, d), im.Block8.empty(d, 128))
    im.rms_norm(xl, None, yl, rl, residual=xl, y8=l8)
    assert torch.equal(y[tail], yl) and torch.equal(rstd[tail], rl) and torch.equal(h[tail], xl + xl)
    assert torch.equal(x8.q[tail].view(torch.uint8), l8.q.view(torch.uint8))
    im.rms_norm_grad(y, h, None, rstd, y)
    im.rms_norm_grad(yl, h[tail], None, rl, yl)
    assert torch.equal(y[tail], yl)
    im.block8_store(x, x8, xt)
    im.block8_store(xl, l8, lt)
    assert torch.equal(x8.q[tail].view(torch.uint8), l8.q.view(torch.uint8))
    assert torch.equal(xt.q[:, -128:].view(torch.uint8), lt.q.view(torch.uint8))
    assert torch.equal(xt.scale[:, -1], lt.scale[:, 0])
    im.block8_load(x8, y)
    assert torch.equal(y, x)
    # whole numbers: exact in any order
    w8 = im.Block8.empty(d, d, 128)
    im.block8_store(torch.eye(d, device="cuda"), w8)
    im.linear8(x8, w8, None, y)
    assert torch.equal(y, x)
    del h, x8, xt
    # two steps of 2.2 GB
    s = x.view(2, n // 2, d)
    out = torch.zeros_like(s)
    im.gated_scan(s, s, out)
    last = s[:, -2:].contiguous()
    want = torch.zeros_like(last)
    im.gated_scan(last, last, want)
    assert torch.equal(out[:, -2:], want)


# ---------------------------------------------------------- differences, graphs
def test_gradients_against_differences():
    """The norm's and the scan's gradients against central differences of the kernels' own
    outputs in fp32, at steps where a difference's rounding is below a thousandth."""
    g = _gen(11)
    n, d, T = 2, 24, 35
    x, gamma, w = torch.randn(n, d, generator=g), 1 + 0.1 * torch.randn(d, generator=g), torch.randn(n, d, generator=g)

    def loss(v):
        y = torch.zeros(n, d, device="cuda")
        im.rms_norm(v.cuda(), gamma.cuda(), y, eps=1e-6)
        return float((y.double() * w.cuda().double()).sum())

    rstd, y = torch.zeros(n, device="cuda"), torch.zeros(n, d, device="cuda")
    im.rms_norm(x.cuda(), gamma.cuda(), y, rstd, 1e-6)
    dx = torch.zeros(n, d, device="cuda")
    im.rms_norm_grad(w.cuda(), x.cuda(), gamma.cuda(), rstd, dx)
    for k in range(5):
        v = torch.randn(n, d, generator=g)
        e = 2.0 ** -7
        num = (loss(x + e * v) - loss(x - e * v)) / (2 * e)
        ana = float((dx.cpu().double() * v.double()).sum())
        # third derivatives e^2 / 6, and roundings of about 40 2^-24 of |y w| over 2 e
        assert abs(num - ana) <= 2e-3 * float((dx.cpu().abs() * v.abs()).sum())

    gate, xs, dh, flags, c0, dc = _scan_case(T, 3, 10, "f32", True, True, 9)

    def total(gv, xv, cv):
        h, out = torch.zeros(T, 3, 10, device="cuda"), torch.zeros(3, 10, device="cuda")
        im.gated_scan(gv.cuda(), xv.cuda(), h, cv.cuda(), out, None, flags[0].cuda(), flags[1].cuda())
        return float((h.double().cpu() * dh.double()).sum() + (out.double().cpu() * dc.double()).sum())

    h, keep = torch.zeros(T, 3, 10, device="cuda"), torch.zeros(3, 3, 10, device="cuda")
    im.gated_scan(gate.cuda(), xs.cuda(), h, c0.cuda(), None, keep, flags[0].cuda(), flags[1].cuda())
    dgate, dxs, ds = torch.zeros_like(h), torch.zeros_like(h), torch.zeros(3, 10, device="cuda")
    im.gated_scan_grad(dh.cuda(), gate.cuda(), xs.cuda(), keep, dgate, dxs, dc.cuda(), ds, flags[0].cuda(),
                       flags[1].cuda())
    for k in range(5):
        vs = [torch.randn(t.shape, generator=g) for t in (gate, xs, c0)]
        e = 2.0 ** -7
        num = (total(gate + e * vs[0], xs + e * vs[1], c0 + e * vs[2]) -
               total(gate - e * vs[0], xs - e * vs[1], c0 - e * vs[2])) / (2 * e)
        ana = sum(float((a.cpu().double() * v.double()).sum()) for a, v in zip((dgate, dxs, ds), vs))
        size = sum(float((a.cpu().abs() * v.abs()).sum()) for a, v in zip((dgate, dxs, ds), vs))
        assert abs(num - ana) <= 2e-3 * size
