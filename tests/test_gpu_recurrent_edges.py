"""Calls of a recurrent policy's blocks that their documentation allows beside the usual ones: outputs
alone in a given workspace, outputs in the place of inputs, other layouts of flags."""
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


def _np(t):
    return t.detach().float().cpu().double().numpy()


@pytest.mark.parametrize("n,i,o", [(1000, 1024, 1024), (1024, 1024, 1024), (40, 361, 69)])
def test_linear8_grad_outputs_alone_in_the_layers_workspace(n, i, o):
    g = _gen(n, i, o)
    dy, x, w = (torch.randn(*z, generator=g).cuda() for z in ((n, o), (n, i), (o, i)))
    xt, wt = im.Block8.empty(i, n), im.Block8.empty(i, o, 128)
    im.block8_store(x, None, xt)
    im.block8_store(w, None, wt)
    ws = im.linear8_grad_workspace(n, i, o)
    outs = [torch.zeros(*z, device="cuda") for z in ((n, i), (o, i), (o,))]
    im.linear8_grad(dy, xt, wt, *outs, workspace=ws)
    for k in range(3):
        one = [torch.full_like(t, 7.0) if j == k else None for j, t in enumerate(outs)]
        im.linear8_grad(dy, xt, wt, *one, workspace=ws)
        assert torch.equal(one[k], outs[k])


@pytest.mark.parametrize("most,calls", [
    ((1000, 65, 1024), [(1000, 65, 1024), (1000, 64, 1024), (999, 3, 1000), (70, 1, 1), (64, 65, 1024)]),
    ((2112, 32, 512), [(2112, 32, 512), (2048, 32, 512), (2111, 31, 511), (1, 32, 512)])])
def test_a_scans_workspace_serves_smaller_calls(most, calls):
    """One workspace for the largest sizes, none of it written behind its end."""
    ws = im.gated_scan_workspace(*most)
    room = torch.full((ws.numel() + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    ws, behind = room[:ws.numel()], room[ws.numel():]
    for T, n, d in calls:
        g = torch.Generator(device="cuda")
        g.manual_seed(T + n + d)
        gate, x, dh = (torch.randn(T, n, d, device="cuda", generator=g) for _ in range(3))
        got = []
        for w in (ws, None):
            h, dgate, dx = (torch.zeros_like(x) for _ in range(3))
            keep = torch.zeros(-(-T // 16), n, d, device="cuda")
            out, dst = torch.zeros(n, d, device="cuda"), torch.zeros(n, d, device="cuda")
            im.gated_scan(gate, x, h, None, out, keep, workspace=w)
            im.gated_scan_grad(dh, gate, x, keep, dgate, dx, None, dst, workspace=w)
            got.append((h, out, keep, dgate, dx, dst))
        assert all(torch.equal(a, b) for a, b in zip(*got))
    assert (behind == 0xA5).all()


@pytest.mark.parametrize("n,i,o", [(200, 2048, 2304), (400, 2048, 2304), (4100, 1408, 1536), (16500, 1536, 2048)])
def test_linear8_grad_of_wide_layers(n, i, o):
    """Whole numbers, exact in fp32, at widths where parts of the larger tiles come to less than 400."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    dy, x, w = (torch.randint(-7, 8, z, device="cuda", generator=g).float() for z in ((n, o), (n, i), (o, i)))
    xt, wt = im.Block8.empty(i, n), im.Block8.empty(i, o, 128)
    im.block8_store(x, None, xt)
    im.block8_store(w, None, wt)
    dx, dw, db = (torch.zeros(*z, device="cuda") for z in ((n, i), (o, i), (o,)))
    im.linear8_grad(dy, xt, wt, dx, dw, db)
    assert torch.equal(dx, (dy.double() @ w.double()).float())
    assert torch.equal(dw, (dy.double().t() @ x.double()).float())
    assert torch.equal(db, dy.double().sum(0).float())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad", [(1, 1, 0), (40, 7, 1), (300, 30, 0), (4097, 361, 0), (300, 513, 0), (301, 1024, 8),
                                     (77, 2047, 1), (41, 4099, 0), (40, 8185, 0), (41, 8191, 1), (40, 8192, 0)])
def test_rms_norm_grad_in_place(n, d, pad, dtype):
    """dx in the place of dy, h or dh, alone and beside dgamma, at widths whose last two pieces share
    columns and lie in one wavefront or in two: the bits of an array of its own."""
    g = _gen(n, d)

    def rows(x):
        wide = torch.full((n, d + pad), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, :d] = x.cuda()
        return wide[:, :d]

    src = [torch.randn(n, d, generator=g).to(DT[dtype]) for _ in range(3)]
    gamma, rstd = (1 + 0.3 * torch.randn(d, generator=g)).cuda(), (0.5 + torch.rand(n, generator=g)).cuda()
    for res in (False, True):
        dy, h, dh = (rows(x) for x in src)
        want, sums = torch.zeros(n, d, dtype=DT[dtype], device="cuda"), torch.zeros(d, device="cuda")
        im.rms_norm_grad(dy, h, gamma, rstd, want, sums, dh if res else None)
        for place in range(3 if res else 2):
            for with_sums in (False, True):
                arrays = [rows(x) for x in src]
                got = torch.zeros(d, device="cuda") if with_sums else None
                im.rms_norm_grad(arrays[0], arrays[1], gamma, rstd, arrays[place], got, arrays[2] if res else None)
                assert torch.equal(arrays[place], want), (res, place)
                assert not with_sums or torch.equal(got, sums)
                for k in range(3):
                    assert k == place or torch.equal(arrays[k].cpu(), src[k])
                if pad:
                    assert torch.isnan(arrays[place]._base[:, d:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,n,d", [(1, 5, 9), (20, 7, 33), (33, 3, 256), (16, 64, 128), (700, 2, 40), (3000, 1, 130)])
def test_flags_of_wider_rows(T, n, d, dtype):
    """Flags as columns of wider rows (as the rollout storage has them), both, either, and as bool, forward
    and backward, with wavefronts of one env and of several."""
    g = _gen(T, n, d)
    gate = (2 + 2 * torch.randn(T, n, d, generator=g)).to(DT[dtype])
    x, dh = (torch.randn(T, n, d, generator=g).to(DT[dtype]) for _ in range(2))
    flags = (torch.rand(2, T, n, generator=g) < 0.15).to(torch.uint8) * 2
    c0, dc = torch.randn(n, d, generator=g), torch.randn(n, d, generator=g)
    wide = torch.full((2, T, n + 5), 0xFF, dtype=torch.uint8, device="cuda")
    wide[:, :, :n] = flags.cuda()
    f = wide[0, :, :n], wide[1, :, :n]
    only = torch.full((T, n + 5), True, device="cuda")
    only[:, :n] = (flags[0] | flags[1]).cuda() != 0
    both, first = (flags[0] | flags[1]).numpy() != 0, flags[0].numpy() != 0
    half = O.HALF[dtype] * 1.01
    for args, end in ((f, both), ((f[0], None), first), ((None, f[0]), first), ((only[:, :n], None), both)):
        h64, before, last, eh, ebefore, elast = O.scan(_np(gate), _np(x), end, _np(c0))
        h, out = torch.zeros_like(x, device="cuda"), torch.zeros(n, d, device="cuda")
        keep = torch.zeros(-(-T // 16), n, d, device="cuda")
        im.gated_scan(gate.cuda(), x.cuda(), h, c0.cuda(), out, keep, *args)
        assert (np.abs(_np(h) - h64) <= eh + half * (np.abs(h64) + eh)).all()
        assert (np.abs(_np(out) - last) <= elast).all()
        dgate, dx = torch.zeros_like(h), torch.zeros_like(h)
        dgate64, dx64, dst64, eg, ex, es = O.scan_grad(_np(dh), _np(gate), _np(x), end, before, ebefore, _np(dc))
        im.gated_scan_grad(dh.cuda(), gate.cuda(), x.cuda(), keep, dgate, dx, dc.cuda(), out, *args)
        assert (np.abs(_np(dgate) - dgate64) <= eg + half * (np.abs(dgate64) + eg)).all()
        assert (np.abs(_np(dx) - dx64) <= ex + half * (np.abs(dx64) + ex)).all()
        assert (np.abs(_np(out) - dst64) <= es).all()
