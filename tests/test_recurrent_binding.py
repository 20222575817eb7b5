"""The binding of a recurrent policy's blocks without a GPU: scratch memory, and the arguments
that it refuses.  Tensors are on the CPU, the device -1 of the calls, and the C entries note
what they are given."""
import weakref
from contextlib import contextmanager

import pytest
import torch

from paper_2609_09821_amd import binding as im

BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


@pytest.fixture
def host(monkeypatch):
    im.lib()
    monkeypatch.setattr(im, "_torch", torch)
    monkeypatch.setattr(im, "_call_stream", lambda stream: (-1, 0))
    monkeypatch.setattr(im, "_space", lambda nbytes: torch.zeros(max(nbytes, 16), dtype=U8))


def _b8(n, d, rows=1):
    return im.Block8.empty(n, d, rows, "cpu")


def _calls():
    """The calls that need scratch memory, as functions of a stream and a workspace."""
    n, i, o, T = 600, 24, 40, 4000
    dy, h = torch.zeros(n, i), torch.zeros(n, i)
    g = torch.zeros(T, 1, i)
    keep = torch.zeros(T // 16, 1, i)
    return [
        lambda **k: im.rms_norm_grad(dy, h, None, torch.zeros(n), None, torch.zeros(i), **k),
        lambda **k: im.linear8_grad(torch.zeros(n, o), _b8(i, n), _b8(i, o, 128), torch.zeros(n, i),
                                    torch.zeros(o, i), torch.zeros(o), **k),
        lambda **k: im.gated_scan(g, g, g, **k),
        lambda **k: im.gated_scan_grad(g, g, g, keep, g, g, **k),
    ]


ENTRIES = ("im_rms_norm_grad", "im_block_linear_grad", "im_gated_scan", "im_gated_scan_grad")


def test_scratch_memory(host, monkeypatch):
    """It comes from the pool of the call's stream and is held until the launch; given memory of
    another layout or device is refused."""
    where, refs, seen = ["torch's own"], [], []

    @contextmanager
    def on(stream):
        before, where[0] = where[0], stream
        yield
        where[0] = before

    def space(nbytes):
        t = torch.zeros(max(nbytes, 16), dtype=U8)
        refs.append((where[0], weakref.ref(t), t.data_ptr()))
        return t

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(im, "_space", space)
    for f in ENTRIES:
        monkeypatch.setattr(im, f, lambda a, raw: seen.append(
            (refs[-1][1]() is not None and a.workspace == refs[-1][2]) if refs else a.workspace))
    for stream, pool in (("side", "side"), (None, "torch's own")):
        for call in _calls():
            call(stream=stream)
            assert refs[-1][0] == pool and seen.pop() is True
            assert refs.pop()[1]() is None and not refs
    for call in _calls():
        with pytest.raises(ValueError, match="workspace"):
            call(workspace=torch.zeros(1 << 22, dtype=U8)[::2])
        ws = torch.zeros(1 << 22, dtype=U8)
        call(workspace=ws)
        assert seen.pop() == ws.data_ptr()


def test_calls_on_no_rows(host):
    x, v = torch.zeros(0, 24, dtype=BF16), torch.zeros(0)
    c = _b8(0, 24)
    im.block8_store(x, c)
    im.block8_load(c, x)
    im.rms_norm(x, None, x, v, residual=x, h=torch.zeros(0, 24, dtype=BF16), y8=c)
    im.rms_norm_grad(x, x, None, v, x)
    im.linear8(c, _b8(40, 24, 128), None, torch.zeros(0, 40))
    im.linear8_grad(torch.zeros(0, 40, dtype=BF16), None, _b8(24, 40, 128), x)
    e = torch.zeros(3, 0, 24)
    im.gated_scan(e, e, e, e[0], e[0])
    im.gated_scan_grad(e, e, e, torch.zeros(1, 0, 24), e, e)


def _x(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype)


@pytest.mark.parametrize("call,words", [
    (lambda: im.block8_store(_x(4, 8), _b8(4, 9)), "rows of 9"),
    (lambda: im.block8_store(_x(4, 8), _b8(3, 8)), "c.q must be"),
    (lambda: im.block8_store(_x(4, 8, dtype=torch.float16), _b8(4, 8)), "float32 or bfloat16"),
    (lambda: im.block8_store(_x(8, 4).t(), _b8(4, 8)), "lie together"),
    (lambda: im.block8_store(_x(4, 8), None, _b8(4, 8)), "t holds|rows of"),
    (lambda: im.block8_store(_x(4, 8), im.Block8(_x(4, 128, dtype=U8), _x(4, 1, dtype=U8), 8)), "c.q must"),
    (lambda: im.block8_store(_x(4, 8), im.Block8(_b8(4, 8).q, _x(4, 1, dtype=U8), 8, 64)), "rows must"),
    (lambda: im.block8_store(_x(300, 8), im.Block8(_b8(300, 8).q, _x(300, 1, dtype=U8), 8, 128)), "c.scale"),
    (lambda: im.rms_norm(_x(4, 8), _x(7), _x(4, 8)), "gamma"),
    (lambda: im.rms_norm(_x(4, 8), None, _x(4, 8, dtype=BF16)), "y must be"),
    (lambda: im.rms_norm(_x(4, 8), None, _x(4, 8), residual=_x(3, 8)), "residual"),
    (lambda: im.rms_norm(_x(4, 8), None, _x(4, 8), _x(5)), "rstd"),
    (lambda: im.rms_norm_grad(_x(4, 8), _x(4, 8, dtype=BF16), None, _x(4), _x(4, 8)), "h must be"),
    (lambda: im.rms_norm_grad(_x(4, 8), _x(4, 8), None, _x(4), _x(4, 8), dh=_x(4, 9)), "dh must be"),
    (lambda: im.linear8(_b8(4, 8), _b8(16, 9, 128), None, _x(4, 16)), "rows of 9"),
    (lambda: im.linear8(_b8(4, 8), _b8(16, 8, 128), _x(15), _x(4, 16)), "bias"),
    (lambda: im.linear8(_b8(4, 8), _b8(16, 8, 128), None, _x(4, 15)), "y must be"),
    (lambda: im.linear8_grad(_x(4, 16), _b8(8, 4), _b8(8, 15, 128), _x(4, 8)), "rows of 15"),
    (lambda: im.linear8_grad(_x(4, 16), _b8(8, 5), None, None, _x(16, 8)), "rows of 5"),
    (lambda: im.linear8_grad(_x(4, 16), _b8(8, 4), None, None, _x(15, 8)), "dw must be"),
    (lambda: im.linear8_grad(_x(4, 16), None, None, db=_x(16), y=_x(4, 16, dtype=BF16)), "y must be"),
    (lambda: im.gated_scan(_x(3, 4, 8), _x(3, 4, 8, dtype=BF16), _x(3, 4, 8)), "gate must be"),
    (lambda: im.gated_scan(_x(3, 4, 8), _x(3, 4, 8), _x(3, 4, 9)), "h must be"),
    (lambda: im.gated_scan(_x(3, 4, 16)[..., ::2], _x(3, 4, 8), _x(3, 4, 8)), "lie together"),
    (lambda: im.gated_scan(*[_x(3, 4, 8)] * 3, _x(8, 4)), "state must be"),
    (lambda: im.gated_scan(*[_x(3, 4, 8)] * 3, _x(4, 8, dtype=BF16)), "state"),
    (lambda: im.gated_scan(*[_x(3, 4, 8)] * 3, keep=_x(2, 4, 8)), "keep"),
    (lambda: im.gated_scan(*[_x(3, 4, 8)] * 3, terminated=_x(3, 4)), "uint8 or bool"),
    (lambda: im.gated_scan(*[_x(3, 4, 8)] * 3, terminated=_x(3, 5, dtype=U8)), "terminated must"),
    (lambda: im.gated_scan(*[_x(3, 4, 8)] * 3, terminated=_x(3, 4, dtype=U8),
                           truncated=_x(3, 9, dtype=U8)[:, :4]), "same row stride"),
    (lambda: im.gated_scan(_x(3, 4, 8), _x(3, 4, 8), _x(1, 4, 8).expand(3, 4, 8)), "overlap"),
    (lambda: im.gated_scan_grad(*[_x(3, 4, 8)] * 3, _x(2, 4, 8), *[_x(3, 4, 8)] * 2), "keep"),
    (lambda: im.gated_scan_grad(*[_x(3, 4, 8)] * 3, _x(1, 4, 8), _x(3, 4, 8), _x(3, 4, 8), _x(4, 7)), "dstate"),
])
def test_refused_arguments(host, call, words):
    with pytest.raises((ValueError, im.ImError), match=words):
        call()
