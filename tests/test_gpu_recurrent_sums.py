"""Products in 8 bits on the GPU: every sum is one of fp32, whatever the output's type and the tile.

The products are multiples of 2^-5 that e4m3 holds at scale 2^0, all sums below 2^18: fp32's 24
bits form them exactly in any order, so that outputs have to be equal, bit for bit, to the exact sum
rounded once.  Products of 448 by 448 stand among products of single digits, and cancel."""
import zlib

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2609_09821_amd import binding as im  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def _gen(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


def _values(n, k, unit, pairs, g):
    """[n][k] of -15 .. 15 units; of each 128 columns two hold 448, the second one -448 where `pairs`
    (rows by the other operand's then cancel).  e4m3 holds them exactly."""
    x = torch.randint(-15, 16, (n, k), device="cuda", generator=g).float() * unit
    for c in range(0, k, 128):
        width = min(128, k - c)
        if width > 8:
            x[:, c + width // 3] = 448.0
            x[:, c + width - 2] = -448.0 if pairs else 448.0
    return x


def _stored(x, rows, t=False):
    b = im.Block8.empty(*(x.shape[::-1] if t else x.shape), rows)
    im.block8_store(x, None if t else b, b if t else None)
    back = torch.zeros(b.shape, device="cuda")
    im.block8_load(b, back)
    assert torch.equal(back, x.t() if t else x)
    return b


# rows, in and out of every kind of tile, with one to nine blocks of k and ends in both directions
SIZES = [(1, 361, 1024), (5, 1100, 40), (64, 1152, 300), (200, 700, 150), (2048, 1024, 1024), (4200, 1100, 1100),
         (16384, 1024, 1024), (16500, 1100, 1030), (65601, 300, 69), (66000, 1000, 897)]


@pytest.mark.parametrize("n,i,o", SIZES)
def test_linear8_sums_are_of_fp32(n, i, o):
    g = _gen(n, i, o)
    x, w = _values(n, i, 2.0 ** -2, True, g), _values(o, i, 2.0 ** -3, False, g)
    x8, w8 = _stored(x, 1), _stored(w, 128)
    bias = torch.randint(-99, 100, (o,), device="cuda", generator=g).float()
    want = x.double() @ w.double().t() + bias.double()
    assert float(want.abs().max()) < 2.0 ** 18
    want = want.float()
    for dt in (F32, BF16):
        y = torch.full((n + 1, o), 7.0, dtype=dt, device="cuda")
        im.linear8(x8, w8, bias, y[:n])
        assert torch.equal(y[:n], want.to(dt)) and (y[n] == 7).all()
    # 8 bits, alone and beside y: those of the sum
    stored = im.Block8.empty(n, o)
    im.block8_store(want, stored)
    for dt in (None, BF16, F32):
        y = None if dt is None else torch.zeros(n, o, dtype=dt, device="cuda")
        y8 = im.Block8.empty(n, o)
        im.linear8(x8, w8, bias, y, y8=y8)
        assert torch.equal(y8.q.view(torch.uint8), stored.q.view(torch.uint8))
        assert torch.equal(y8.scale, stored.scale)
        assert dt is None or torch.equal(y, want.to(dt))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("n,i,o", [(1, 40, 300), (130, 361, 700), (1024, 1024, 1024), (4095, 361, 1024),
                                   (16500, 1030, 520), (65601, 513, 260)])
def test_linear8_grad_sums_are_of_fp32(n, i, o, dt):
    g = _gen(n, i, o, 1)
    dy, w = _values(n, o, 2.0 ** -2, True, g), _values(i, o, 2.0 ** -3, False, g)
    # along the rows too the blocks of dy hold 448, so that both ways are exact
    wt = _stored(w, 128)
    xt = im.Block8.empty(i, n)
    x = torch.randint(-7, 8, (n, i), device="cuda", generator=g).float()
    im.block8_store(x, None, xt)
    dx, dw, db = (torch.zeros(n, i, dtype=dt, device="cuda"), torch.zeros(o, i, device="cuda"),
                  torch.zeros(o, device="cuda"))
    im.linear8_grad(dy.to(dt), xt, wt, dx, dw, db)
    assert torch.equal(dx, (dy.double() @ w.double().t()).float().to(dt))
    # multiples of 2^-2 below 2^22, and those of the columns of 448: of 2^6 below 2^30
    assert torch.equal(dw, (dy.double().t() @ x.double()).float())
    assert torch.equal(db, dy.double().sum(0).float())


def test_linear8_of_normal_values_to_bf16():
    """An output in bf16 is the one in fp32, rounded."""
    n, i, o = 4096, 1024, 1024
    g = _gen(0)
    x8, w8 = im.Block8.empty(n, i), im.Block8.empty(o, i, 128)
    im.block8_store(torch.randn(n, i, device="cuda", generator=g), x8)
    im.block8_store(torch.randn(o, i, device="cuda", generator=g), w8)
    x, w = torch.zeros(n, i, device="cuda"), torch.zeros(o, i, device="cuda")
    im.block8_load(x8, x)
    im.block8_load(w8, w)
    want = x.double() @ w.double().t()
    y32, y16 = torch.zeros(n, o, device="cuda"), torch.zeros(n, o, dtype=BF16, device="cuda")
    im.linear8(x8, w8, None, y32)
    im.linear8(x8, w8, None, y16)
    # products are exact; sums of i in any order, each off by a step of 2^-23 at most
    mass = x.double().abs() @ w.double().abs().t()
    assert bool(((y32.double() - want).abs() <= i * 2.0 ** -23 * mass).all())
    assert torch.equal(y16, y32.to(BF16))
