"""The layers of experts' C ABI without a GPU: what the calls refuse before they touch the
device, and the workspace sizes."""
import ctypes as C
import os

import pytest

from paper_2609_09821_amd import binding as im

P = 1 << 20      # stands for a device address that no refused call reads


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(im.LIB_PATH):
        from paper_2609_09821_amd import build
        build.build()
    return im.lib()


def _refused(lib, status, code, words):
    assert status == code, (status, lib.im_last_error())
    assert words in lib.im_last_error().decode(), lib.im_last_error()


BAD, UNS = im.IM_ERR_INVALID_ARG, im.IM_ERR_UNSUPPORTED


@pytest.mark.parametrize("args,code,words", [
    ((P, -1, 4, P, P, P, 1 << 20), BAD, "n must"),
    ((P, 10, 0, P, P, P, 1 << 20), BAD, "n must"),
    ((P, (1 << 30) + 1, 4, P, P, P, 1 << 20), UNS, "2^30"),
    ((P, 10, 1025, P, P, P, 1 << 20), UNS, "IM_MAX_EXPERTS"),
    ((None, 10, 4, P, P, P, 1 << 20), BAD, "NULL"),
    ((P, 10, 4, None, P, P, 1 << 20), BAD, "NULL"),
    ((P, 10, 4, P, None, P, 1 << 20), BAD, "NULL"),
    ((P, 1 << 20, 4, P, P, None, 1 << 20), BAD, "workspace"),
    ((P, 1 << 20, 4, P, P, P, 8), BAD, "workspace"),
    ((P, 1 << 20, 4, P, P, P + 2, 1 << 20), BAD, "aligned"),
])
def test_group_rows_refuses(lib, args, code, words):
    _refused(lib, lib.im_group_rows(*args, None), code, words)


@pytest.mark.parametrize("n,d,ld,dtype,ck,x,code,words", [
    (-1, 8, 8, 0, (P, P, 8, 1), P, BAD, "n must"),
    (4, 0, 8, 0, (P, P, 8, 1), P, BAD, "width"),
    (4, 8, 7, 0, (P, P, 8, 1), P, BAD, "ld_x"),
    (4, 8, 8, 2, (P, P, 8, 1), P, BAD, "dtype"),
    (4, 8, 8, 1, (P, P, 7, 1), P, BAD, "ld_q"),
    (4, 33, 33, 1, (P, P, 33, 1), P, BAD, "ld_scale"),
    (4, 8, 8, 1, (None, P, 8, 1), P, BAD, "NULL checkpoint"),
    (4, 8, 8, 1, (P, None, 8, 1), P, BAD, "NULL checkpoint"),
    (4, 8, 8, 1, (P, P, 8, 1), None, BAD, "NULL x"),
    ((1 << 30) + 1, 8, 8, 1, (P, P, 8, 1), P, UNS, "2^30"),
])
def test_checkpoint_refuses(lib, n, d, ld, dtype, ck, x, code, words):
    c = im.ImCheckpoint(*ck)
    _refused(lib, lib.im_checkpoint_store(x, ld, dtype, n, d, C.byref(c), None), code, words)
    _refused(lib, lib.im_checkpoint_load(C.byref(c), n, d, x, ld, dtype, None), code, words)


def test_null_structs(lib):
    for f in (lib.im_layer_norm, lib.im_layer_norm_grad, lib.im_expert_linear, lib.im_expert_linear_grad):
        _refused(lib, f(None, None), BAD, "NULL im_")
    _refused(lib, lib.im_checkpoint_store(P, 8, 0, 4, 8, None, None), BAD, "NULL checkpoint")


def _norm(**over):
    a = im.ImNorm(4, 8, 0, 1e-5, P, 8, P, P, P, 8, P, P, None)
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,code,words", [
    (dict(n=-1), BAD, "n must"), (dict(d=0), BAD, "width"), (dict(d=8193, ld_x=9000, ld_y=9000), UNS, "WIDTH"),
    (dict(eps=-1.0), BAD, "eps"), (dict(eps=float("nan")), BAD, "eps"), (dict(dtype=7), BAD, "dtype"),
    (dict(ld_x=7), BAD, "ld_x"), (dict(ld_y=7), BAD, "ld_y"), (dict(x=None), BAD, "NULL x"),
    (dict(y=None), BAD, "NULL x or y"),
    (dict(checkpoint=C.pointer(im.ImCheckpoint(P, P, 4, 1))), BAD, "ld_q"),
])
def test_layer_norm_refuses(lib, over, code, words):
    _refused(lib, lib.im_layer_norm(C.byref(_norm(**over)), None), code, words)


def _norm_grad(**over):
    a = im.ImNormGrad(4, 8, 0, P, 8, P, 8, None, P, P, P, P, 8, P, P, P, 1 << 20)
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,code,words", [
    (dict(n=-1), BAD, "n must"), (dict(d=8193), UNS, "WIDTH"), (dict(ld_dy=7), BAD, "ld_dy"),
    (dict(ld_x=7), BAD, "ld_x"), (dict(ld_dx=7), BAD, "ld_dx"), (dict(dy=None), BAD, "NULL dy"),
    (dict(mean=None), BAD, "mean"), (dict(rstd=None), BAD, "rstd"), (dict(x=None), BAD, "neither x"),
    (dict(dx=None, dgamma=None, dbeta=None), BAD, "no output"), (dict(workspace=None), BAD, "workspace"),
    (dict(workspace_bytes=63), BAD, "workspace"),
    (dict(x=None, checkpoint=C.pointer(im.ImCheckpoint(P, P, 8, 0))), BAD, "ld_scale"),
])
def test_layer_norm_grad_refuses(lib, over, code, words):
    _refused(lib, lib.im_layer_norm_grad(C.byref(_norm_grad(**over)), None), code, words)


def _layer(**over):
    a = im.ImExpertLayer(4, 2, 8, 16, 1, 1, 0, P, P, P, 8, P, 8, P, P, 16)
    for k, v in over.items():
        setattr(a, k, v)
    return a


LAYER = [
    (dict(n=-1), BAD, "n must"), (dict(in_=0), BAD, "width"), (dict(out=0), BAD, "out"),
    (dict(n_experts=0), BAD, "n_experts"), (dict(n_experts=1025), UNS, "IM_MAX_EXPERTS"),
    (dict(n=(1 << 30) + 1), UNS, "2^30"), (dict(dtype=0), UNS, "bf16 only"), (dict(dtype=5), BAD, "dtype"),
    (dict(offsets=None), BAD, "offsets"), (dict(ld_x=7), BAD, "ld_x"), (dict(ld_w=7), BAD, "ld_w"),
    (dict(in_=1 << 15, out=(1 << 15) + 1), UNS, "2^30"), (dict(n=1 << 30, out=1 << 10), UNS, "tiles"),
]


@pytest.mark.parametrize("over,code,words", LAYER + [
    (dict(y_dtype=3), BAD, "y_dtype"), (dict(ld_y=15), BAD, "ld_y"), (dict(x=None), BAD, "NULL x"),
    (dict(w=None), BAD, "NULL x, w"), (dict(y=None), BAD, "or y"),
])
def test_expert_linear_refuses(lib, over, code, words):
    _refused(lib, lib.im_expert_linear(C.byref(_layer(**over)), None), code, words)


def _layer_grad(**over):
    a = im.ImExpertLayerGrad(4, 2, 8, 16, 1, 0, P, P, P, 16, P, 8, None, P, 8, P, 8, P, 8, P, P, 1 << 20)
    for k, v in over.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("over,code,words", LAYER + [
    (dict(ld_dy=15), BAD, "ld_dy"), (dict(ld_dx=7), BAD, "ld_dx"), (dict(ld_dw=7), BAD, "ld_dw"),
    (dict(dy=None), BAD, "NULL dy"), (dict(w=None), BAD, "NULL dy or w"), (dict(x=None), BAD, "neither x"),
    (dict(dx=None, dw=None, db=None), BAD, "no output"), (dict(workspace=None), BAD, "workspace"),
    (dict(workspace_bytes=100), BAD, "workspace"), (dict(workspace=P + 4), BAD, "aligned"),
    (dict(x=None, relu_x=1, dw=None, db=None), BAD, "neither x"),
    (dict(x=None, checkpoint=C.pointer(im.ImCheckpoint(P, P, 7, 1))), BAD, "ld_q"),
])
def test_expert_linear_grad_refuses(lib, over, code, words):
    _refused(lib, lib.im_expert_linear_grad(C.byref(_layer_grad(**over)), None), code, words)


def test_empty_calls_are_done(lib):
    """Nothing to compute and nothing to write: no launch, no device needed."""
    c = im.ImCheckpoint(None, None, 8, 1)
    assert lib.im_checkpoint_store(None, 8, 0, 0, 8, C.byref(c), None) == im.IM_OK
    assert lib.im_layer_norm(C.byref(_norm(n=0, x=None, y=None)), None) == im.IM_OK
    assert lib.im_layer_norm_grad(C.byref(_norm_grad(n=0, dgamma=None, dbeta=None)), None) == im.IM_OK
    assert lib.im_expert_linear(C.byref(_layer(n=0, x=None, w=None, y=None)), None) == im.IM_OK
    assert lib.im_expert_linear_grad(C.byref(_layer_grad(n=0, dw=None, db=None)), None) == im.IM_OK


def test_workspace_sizes(lib):
    """Sizes out of range have no workspace; sizes in range one that covers the documented parts."""
    assert lib.im_group_rows_workspace(-1, 4) == -1
    assert lib.im_group_rows_workspace(5, 0) == -1
    assert lib.im_group_rows_workspace(5, 1025) == -1
    assert lib.im_group_rows_workspace(1 << 20, 1024) > 0
    assert lib.im_layer_norm_grad_workspace(1, 8193) == -1
    assert lib.im_layer_norm_grad_workspace(-1, 8) == -1
    assert lib.im_layer_norm_grad_workspace(0, 8) >= 2 * 8 * 4
    assert lib.im_expert_linear_grad_workspace(5, 2, 0, 8) == -1
    assert lib.im_expert_linear_grad_workspace(5, 2, 8, (1 << 20) + 1) == -1
    assert lib.im_expert_linear_grad_workspace(0, 2, 8, 8) >= 0
    assert lib.im_expert_linear_grad_workspace(1 << 20, 16, 1024, 1024) >= 16 * 4 * 1024 * 1024
