"""The layers of experts' binding without a GPU: the calls' scratch memory.  Tensors are on the
CPU, the device -1 of the calls, and the C entries note what they are given."""
import weakref
from contextlib import contextmanager

import pytest
import torch

from paper_2609_09821_amd import binding as im


@pytest.fixture
def calls(monkeypatch):
    """The three calls that need scratch memory, as functions of a stream and a workspace, and
    what became of each: (torch's stream when its memory was allocated, addresses in use)."""
    if not im._lib:
        im.lib()
    current, allocated, used = ["torch's own"], [], []

    @contextmanager
    def on(stream):
        before, current[0] = current[0], stream
        yield
        current[0] = before

    def space(nbytes):
        t = torch.zeros(max(nbytes, 16), dtype=torch.uint8)
        t.record_stream = lambda s: None
        allocated.append((current[0], t))
        return t

    monkeypatch.setattr(im, "_torch", torch)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(im, "_call_stream", lambda stream: (-1, 0))
    monkeypatch.setattr(im, "_space", space)
    monkeypatch.setattr(im, "im_group_rows", lambda *a: used.append(a[5]))
    for f in ("im_layer_norm_grad", "im_expert_linear_grad"):
        monkeypatch.setattr(im, f, lambda a, raw: used.append(a.workspace))

    n, e, i, o = 6000, 4, 24, 40
    idx = dict(dtype=torch.int32)
    off, rows = torch.zeros(e + 1, **idx), torch.zeros(n, **idx)
    x, dy = torch.zeros(n, i, dtype=torch.bfloat16), torch.zeros(n, o, dtype=torch.bfloat16)
    w = torch.zeros(e, o, i, dtype=torch.bfloat16)
    stat, dg = torch.zeros(n), torch.zeros(i)
    return [
        lambda **k: im.group_rows(torch.zeros(n, **idx), off, rows, **k),
        lambda **k: im.layer_norm_grad(x, x, None, stat, stat, None, dg, **k),
        lambda **k: im.expert_linear_grad(dy, x, w, off, rows, dw=torch.zeros(e, o, i), **k),
    ], allocated, used


def test_scratch_memory_is_of_the_calls_stream(calls):
    """Memory of another stream's pool may still be in use by that stream's work."""
    calls, allocated, used = calls
    for stream, where in (("side", "side"), (None, "torch's own")):
        for call in calls:
            call(stream=stream)
            at, t = allocated.pop()
            assert at == where and not allocated
            assert used.pop() == t.data_ptr()


def test_scratch_memory_is_held_until_the_launch(calls, monkeypatch):
    """Freed before, another thread could be given it between the two."""
    calls, allocated, used = calls
    refs, alive = [], []

    def space(nbytes):
        t = torch.zeros(max(nbytes, 16), dtype=torch.uint8)
        refs.append(weakref.ref(t))
        return t

    monkeypatch.setattr(im, "_space", space)
    for f in ("im_group_rows", "im_layer_norm_grad", "im_expert_linear_grad"):
        monkeypatch.setattr(im, f, lambda *a: alive.append(refs[-1]() is not None))
    for stream in ("side", None):
        for call in calls:
            call(stream=stream)
    assert alive == [True] * 6
    assert all(r() is None for r in refs)


class _OnDevice(torch.Tensor):
    """Memory that says it is on device 1."""
    is_cuda = True

    def get_device(self):
        return 1


def test_a_workspace_of_another_device_is_refused(calls):
    calls, _, used = calls
    for call in calls:
        with pytest.raises(ValueError, match="workspace"):
            call(workspace=torch.zeros(1 << 20, dtype=torch.uint8).as_subclass(_OnDevice))
        with pytest.raises(ValueError, match="workspace"):
            call(workspace=torch.zeros(1 << 21, dtype=torch.uint8)[::2])
        assert not used
        call(workspace=torch.zeros(1 << 20, dtype=torch.uint8))
        used.clear()


def test_calls_on_no_rows(monkeypatch):
    """An empty batch is done, whichever of the rows' outputs is asked for."""
    im.lib()
    monkeypatch.setattr(im, "_torch", torch)
    monkeypatch.setattr(im, "_call_stream", lambda stream: (-1, 0))
    x, y = (torch.zeros(0, d, dtype=torch.bfloat16) for d in (24, 40))
    w, off = torch.zeros(4, 40, 24, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    stat, ck = torch.zeros(0), im.Checkpoint.empty(0, 24, "cpu")
    im.checkpoint_store(x, ck)
    im.checkpoint_load(ck, x)
    im.layer_norm(x, None, None, x, stat, stat, checkpoint=ck)
    im.expert_linear(x, w, None, off, None, y)
    for src in (x, ck):
        im.layer_norm_grad(x, src, None, stat, stat, dx=x)
        im.expert_linear_grad(y, src, w, off, None, dx=x)
        im.expert_linear_grad(y, src, w, off, off[:0], dx=x, relu_x=True)
