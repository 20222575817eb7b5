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
