"""The C ABI of a recurrent policy's blocks without a GPU: what the calls refuse before they
touch the device, and the workspace sizes."""
import ctypes as C
import os
import random

import pytest

from paper_2609_09821_amd import binding as im

P = 1 << 20      # stands for a device address that no refused call reads
BAD, UNS = im.IM_ERR_INVALID_ARG, im.IM_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(im.LIB_PATH):
        from paper_2609_09821_amd import build
        build.build()
    return im.lib()


def _refused(lib, status, code, words):
    assert status == code, (status, lib.im_last_error())
    assert words in lib.im_last_error().decode(), lib.im_last_error()


def _b8(d=8, n=4, rows=1, **over):
    b = im.ImBlock8(P, P, -(-d // 128) * 128, -(-d // 128), rows)
    for k, v in over.items():
        setattr(b, k, v)
    return b


_HOLD = []


def _held(*a, **k):
    """Address of a matrix in 8 bits that lives as long as the tests."""
    _HOLD.append(_b8(*a, **k))
    return C.addressof(_HOLD[-1])


_SQUARE, _SQUARE16 = _held(rows=128), _held(16, rows=128)
BAD_BLOCKS = [
    (dict(rows=2), "rows must"), (dict(rows=0), "rows must"), (dict(ld_q=112), "ld_q"),
    (dict(ld_q=136), "ld_q"), (dict(ld_scale=0), "ld_scale"), (dict(q=None), "NULL block8"),
    (dict(scale=None), "NULL block8"), (dict(q=P + 8), "aligned"),
]


@pytest.mark.parametrize("over,words", BAD_BLOCKS)
def test_block8_arguments(lib, over, words):
    b = _b8(**over)
    for status in (lib.im_block_store(P, 8, 0, 4, 8, C.byref(b), None, None),
                   lib.im_block_store(P, 4, 0, 8, 4, None, C.byref(b), None),
                   lib.im_block_load(C.byref(b), 4, 8, P, 8, 0, None),
                   lib.im_rms_norm(C.byref(_rms(y8=C.addressof(b))), None),
                   lib.im_block_linear(C.byref(_layer(x=C.addressof(b))), None),
                   lib.im_block_linear(C.byref(_layer(w=C.addressof(b))), None),
                   lib.im_block_linear(C.byref(_layer(out=8, ld_y=8, y8=C.addressof(b))), None),
                   lib.im_block_linear_grad(C.byref(_layer_grad(xt=C.addressof(b))), None),
                   lib.im_block_linear_grad(C.byref(_layer_grad(wt=C.addressof(b))), None)):
        _refused(lib, status, BAD, words)


@pytest.mark.parametrize("x,ld,dtype,n,d,c,t,code,words", [
    (P, 8, 0, -1, 8, _b8(), None, BAD, "n must"),
    (P, 8, 0, 4, 0, _b8(), None, BAD, "width"),
    (P, 8, 2, 4, 8, _b8(), None, BAD, "dtype"),
    (P, 7, 0, 4, 8, _b8(), None, BAD, "ld_x"),
    (None, 8, 0, 4, 8, _b8(), None, BAD, "NULL x"),
    (P, 8, 0, 4, 8, None, None, BAD, "neither"),
    (P, 8, 0, 4, 8, _b8(), _b8(4, rows=128), BAD, "same rows"),
    (P, 8, 0, (1 << 30) + 1, 8, _b8(), None, UNS, "2^30"),
    (P, 1 << 21, 0, 4, (1 << 20) + 1, _b8((1 << 20) + 1), None, UNS, "2^20"),
])
def test_block8_store_refuses(lib, x, ld, dtype, n, d, c, t, code, words):
    ref = [b and C.byref(b) for b in (c, t)]
    _refused(lib, lib.im_block_store(x, ld, dtype, n, d, *ref, None), code, words)
    if c and not t:
        _refused(lib, lib.im_block_load(ref[0], n, d, x, ld, dtype, None), code, words)


def test_null_arguments(lib):
    for f in (lib.im_rms_norm, lib.im_rms_norm_grad, lib.im_block_linear, lib.im_block_linear_grad,
              lib.im_gated_scan, lib.im_gated_scan_grad):
        _refused(lib, f(None, None), BAD, "NULL im_")
    _refused(lib, lib.im_block_load(None, 4, 8, P, 8, 0, None), BAD, "NULL block8")


def _set(a, over):
    for k, v in over.items():
        setattr(a, k, v)
    return a


def _rms(**over):
    return _set(im.ImRms(4, 8, 0, 1e-6, P, 8, P, 8, P, 2 * P, 8, 3 * P, 8, None, P), over)


@pytest.mark.parametrize("over,code,words", [
    (dict(n=-1), BAD, "n must"), (dict(d=0), BAD, "width"), (dict(eps=-1.0), BAD, "eps"),
    (dict(d=8193, ld_x=9000, ld_residual=9000, ld_h=9000, ld_y=9000), UNS, "WIDTH"),
    (dict(eps=float("nan")), BAD, "eps"), (dict(dtype=7), BAD, "dtype"), (dict(ld_x=7), BAD, "ld_x"),
    (dict(ld_residual=7), BAD, "ld_"), (dict(ld_h=7), BAD, "ld_"), (dict(ld_y=7), BAD, "ld_"),
    (dict(x=None), BAD, "NULL x"), (dict(h=None, y=None, rstd=None), BAD, "no output"),
    (dict(h=3 * P), BAD, "one array"), (dict(y8=_SQUARE), BAD, "rows must be 1"),
])
def test_rms_norm_refuses(lib, over, code, words):
    _refused(lib, lib.im_rms_norm(C.byref(_rms(**over)), None), code, words)


def _rms_grad(**over):
    return _set(im.ImRmsGrad(4, 8, 0, P, 8, P, 8, P, 8, P, P, P, 8, P, P, 1 << 20), over)


@pytest.mark.parametrize("over,code,words", [
    (dict(n=-1), BAD, "n must"), (dict(d=0), BAD, "width"), (dict(dtype=3), BAD, "dtype"),
    (dict(ld_dy=7), BAD, "ld_dy"), (dict(ld_h=7), BAD, "ld_"), (dict(ld_dh=7), BAD, "ld_"),
    (dict(ld_dx=7), BAD, "ld_"), (dict(dy=None), BAD, "NULL"), (dict(h=None), BAD, "NULL"),
    (dict(rstd=None), BAD, "NULL"), (dict(dx=None, dgamma=None), BAD, "no output"),
    (dict(workspace=None), BAD, "workspace"), (dict(workspace_bytes=4), BAD, "workspace"),
    (dict(workspace=P + 2), BAD, "aligned"),
])
def test_rms_norm_grad_refuses(lib, over, code, words):
    _refused(lib, lib.im_rms_norm_grad(C.byref(_rms_grad(**over)), None), code, words)


def _layer(**over):
    return _set(im.ImLayer8(4, 8, 16, 0, 1, _held(8), _held(8, 16, 128), P, P, 16, None), over)


@pytest.mark.parametrize("over,code,words", [
    (dict(n=-1), BAD, "n must"), (dict(in_=0), BAD, "width"), (dict(out=0), BAD, "out must"),
    (dict(y_dtype=5), BAD, "dtype"), (dict(ld_y=15), BAD, "ld_y"), (dict(y=None), BAD, "no output"),
    (dict(x=None), BAD, "NULL block8"), (dict(w=None), BAD, "NULL block8"),
    (dict(in_=129), BAD, "ld_q"), (dict(in_=(1 << 20) + 1), UNS, "2^20"), (dict(out=(1 << 20) + 1), UNS, "2^20"),
    (dict(n=(1 << 30) + 1), UNS, "2^30"), (dict(y8=_SQUARE16), BAD, "rows must be 1"),
    (dict(in_=1 << 16, out=1 << 15), UNS, "in * out"),
])
def test_linear8_refuses(lib, over, code, words):
    _refused(lib, lib.im_block_linear(C.byref(_layer(**over)), None), code, words)


def _layer_grad(**over):
    return _set(im.ImLayer8Grad(4, 8, 16, 0, P, 16, P, 16, _held(4), _held(16, rows=128),
                                P, 8, P, 8, P, P, 1 << 30), over)


@pytest.mark.parametrize("over,code,words", [
    (dict(n=-1), BAD, "n must"), (dict(in_=0), BAD, "width"), (dict(out=0), BAD, "out must"),
    (dict(dtype=5), BAD, "dtype"), (dict(ld_dy=15), BAD, "ld_dy"), (dict(ld_y=15), BAD, "ld_"),
    (dict(ld_dx=7), BAD, "ld_"), (dict(ld_dw=7), BAD, "ld_"), (dict(dy=None), BAD, "NULL dy"),
    (dict(xt=None), BAD, "xt"), (dict(wt=None), BAD, "wt"),
    (dict(dx=None, dw=None, db=None), BAD, "no output"), (dict(workspace=None), BAD, "workspace"),
    (dict(workspace_bytes=16), BAD, "workspace"), (dict(workspace=P + 8), BAD, "aligned"),
    (dict(in_=1 << 16, out=1 << 15), UNS, "in * out"),
])
def test_linear8_grad_refuses(lib, over, code, words):
    _refused(lib, lib.im_block_linear_grad(C.byref(_layer_grad(**over)), None), code, words)


def _scan(**over):
    return _set(im.ImScan(6, 4, 8, 0, P, 32, 8, P, 32, 8, P, P, 4, P, P, 32, 8, P, P, P, 1 << 30), over)


def _scan_grad(**over):
    return _set(im.ImScanGrad(6, 4, 8, 0, P, 32, 8, P, 32, 8, P, 32, 8, P, P, 4, P, P, P, 32, 8, P, 32, 8, P,
                              P, 1 << 30), over)


BOTH = [
    (dict(T=-1), BAD, "T and n"), (dict(n=-1), BAD, "T and n"), (dict(d=0), BAD, "T and n"),
    (dict(dtype=2), BAD, "dtype"), (dict(ld_flags=3), BAD, "ld_flags"), (dict(gate=None), BAD, "NULL gate"),
    (dict(x=None), BAD, "NULL"), (dict(st_x=-32), BAD, "negative"), (dict(ld_gate=-8), BAD, "negative"),
    (dict(T=(1 << 30) + 1), UNS, "2^30"), (dict(n=1 << 20, d=1 << 12), UNS, "2^31"),
]


@pytest.mark.parametrize("over,code,words", BOTH + [
    (dict(h=None), BAD, "NULL"), (dict(st_h=31), BAD, "overlap"), (dict(ld_h=7), BAD, "overlap"),
    (dict(st_h=0), BAD, "overlap"), (dict(st_h=8, ld_h=40), BAD, "overlap"), (dict(st_h=-32), BAD, "overlap"),
])
def test_gated_scan_refuses(lib, over, code, words):
    over = dict(over)
    if over.get("gate", P) is None:
        words = "NULL"
    _refused(lib, lib.im_gated_scan(C.byref(_scan(**over)), None), code, words)


@pytest.mark.parametrize("over,code,words", [(o, c, "NULL" if "NULL" in w else w) for o, c, w in BOTH] + [
    (dict(dh=None), BAD, "NULL"), (dict(keep=None), BAD, "NULL"), (dict(dgate=None), BAD, "NULL"),
    (dict(dx=None), BAD, "NULL"), (dict(st_dx=31), BAD, "overlap"), (dict(ld_dgate=7), BAD, "overlap"),
    (dict(st_dh=-1), BAD, "negative"),
])
def test_gated_scan_grad_refuses(lib, over, code, words):
    _refused(lib, lib.im_gated_scan_grad(C.byref(_scan_grad(**over)), None), code, words)


def test_scan_workspace_is_asked_for(lib):
    need = lib.im_gated_scan_workspace(100000, 1, 8)
    assert need > 0
    big = dict(T=100000, n=1, st_gate=8, st_x=8, st_h=8, st_dh=8, st_dgate=8, st_dx=8)
    for over in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 4)):
        for f, a in ((lib.im_gated_scan, _scan), (lib.im_gated_scan_grad, _scan_grad)):
            s = a()
            _set(s, {k: v for k, v in dict(big, **over).items() if hasattr(s, k)})
            _refused(lib, f(C.byref(s), None), BAD, "workspace")


def test_workspace_sizes(lib):
    assert lib.im_rms_norm_grad_workspace(-1, 8) == lib.im_rms_norm_grad_workspace(4, 0) == -1
    assert lib.im_rms_norm_grad_workspace(4, 8193) == -1 and lib.im_rms_norm_grad_workspace(1 << 20, 512) > 0
    for a in ((-1, 8, 8), (4, 0, 8), (4, 8, 0), ((1 << 30) + 1, 8, 8), (4, 1 << 21, 8), (4, 1 << 16, 1 << 15)):
        assert lib.im_block_linear_grad_workspace(*a) == -1
    # dy in 8 bits, twice, with its scales
    assert lib.im_block_linear_grad_workspace(65536, 1024, 512) >= 2 * 65536 * 516
    for a in ((-1, 4, 8), (4, -1, 8), (4, 4, 0), ((1 << 30) + 1, 1, 1), (4, 1 << 20, 1 << 12)):
        assert lib.im_gated_scan_workspace(*a) == -1
    for a in ((0, 0, 1), (1, 65536, 1024), (32, 16384, 256)):
        assert lib.im_gated_scan_workspace(*a) == 0


def test_calls_on_nothing(lib):
    """Empty batches are done without a look at the arrays."""
    none = dict(n=0, x=None, residual=None, gamma=None, h=None, y=None, rstd=None)
    assert lib.im_rms_norm(C.byref(_rms(**none)), None) == im.IM_OK
    assert lib.im_rms_norm_grad(C.byref(_rms_grad(n=0, dy=None, h=None, rstd=None, dgamma=None)), None) == im.IM_OK
    empty = _b8(q=None, scale=None)
    assert lib.im_block_store(None, 8, 0, 0, 8, C.byref(empty), None, None) == im.IM_OK
    assert lib.im_block_load(C.byref(empty), 0, 8, None, 8, 0, None) == im.IM_OK
    assert lib.im_block_linear(C.byref(_layer(n=0, x=C.addressof(empty), y=None)), None) == im.IM_OK
    assert lib.im_block_linear_grad(C.byref(_layer_grad(n=0, dy=None, dw=None, db=None)), None) == im.IM_OK
    assert lib.im_gated_scan(C.byref(_scan(n=0, gate=None, x=None, h=None)), None) == im.IM_OK
    assert lib.im_gated_scan(C.byref(_scan(T=0, gate=None, x=None, h=None, state_out=None)), None) == im.IM_OK
    assert lib.im_gated_scan_grad(C.byref(_scan_grad(n=0, dh=None)), None) == im.IM_OK


@pytest.mark.parametrize("n,i,o", [(1000, 1024, 1024), (1024, 1024, 1024), (1920, 1024, 1024), (40, 361, 69),
                                   (65536, 1024, 512)])
def test_the_layers_workspace_serves_each_output_alone(lib, n, i, o):
    """db alone is asked for without the layer's input width (in = 1, as the binding does): the
    layer's workspace is large enough.  It is misaligned here, which is looked at last."""
    need = lib.im_block_linear_grad_workspace(n, i, o)
    none = dict(dx=None, dw=None, db=None, ld_dy=o, y=None, workspace=P + 8, workspace_bytes=need)
    for over in (dict(db=P, in_=1), dict(db=P, in_=i), dict(dx=P, in_=i, ld_dx=i, wt=_held(o, i, 128)),
                 dict(dw=P, in_=i, ld_dw=i, xt=_held(n, i))):
        a = _layer_grad(**dict(none, n=n, out=o, **over))
        _refused(lib, lib.im_block_linear_grad(C.byref(a), None), BAD, "aligned")


def _asked(lib, f, a):
    """Whether a call without its arrays is refused for its workspace (or for the arrays)."""
    assert f(C.byref(a), None) == BAD
    said = lib.im_last_error().decode()
    assert ("workspace" in said) != ("NULL gate" in said or "NULL dh" in said), said
    return "workspace" in said


def test_a_scans_workspace_serves_smaller_calls(lib):
    """Sized once for the largest T, n and d, as a program does whose batches vary."""
    rng = random.Random(7)

    def log(hi):
        return max(1, int(round(hi ** rng.random())))

    def pair(most, small):
        ws = lib.im_gated_scan_workspace(*most)
        assert 0 <= lib.im_gated_scan_workspace(*small) <= ws <= 5 << 20, (most, small)
        T, n, d = small
        for f, make in ((lib.im_gated_scan, _scan), (lib.im_gated_scan_grad, _scan_grad)):
            s = make()
            over = dict(T=T, n=n, d=d, ld_flags=n, gate=None, workspace_bytes=ws, dh=None)
            over.update({k: n * d for k in ("st_gate", "st_x", "st_h", "st_dh", "st_dgate", "st_dx")})
            over.update({k: d for k in ("ld_gate", "ld_x", "ld_h", "ld_dh", "ld_dgate", "ld_dx")})
            _set(s, {k: v for k, v in over.items() if hasattr(s, k)})
            assert not _asked(lib, f, s), (most, small)

    pair((1000, 65, 1024), (1000, 64, 1024))
    pair((2112, 32, 512), (2048, 32, 512))
    for _ in range(20000):
        most = log(1 << 20), log(4096), log(2048)
        pair(most, tuple(rng.choice((v, rng.randint(1, v), max(1, v - 1))) for v in most))
    # chunks whose length was rounded down the most
    for lanes in (1, 2, 3, 5, 64, 1000, 8192, 32768):
        for q in (32, 48, 64, 1024):
            T = ((q + 1) * 262144 - 1) // lanes
            for n, d in ((lanes, 1), (lanes, 2), (1, 2 * lanes), (1, 2 * lanes - 1)):
                pair((T, n, d), (T, n, d))


def test_workspaces_grow_with_the_rows(lib):
    """A workspace for n rows serves every call on fewer."""
    for i, o in ((1, 1), (361, 1024), (1024, 512), (1024, 1024), (1536, 1408), (2048, 2304), (69, 4096), (3000, 3000)):
        last = 0
        for n in list(range(0, 9000, 37)) + [16384, 30000, 65536, 1 << 20]:
            now = lib.im_block_linear_grad_workspace(n, i, o)
            assert now >= last, (n, i, o)
            last = now
    for d in (1, 30, 361, 512, 1024, 8192):
        sizes = [lib.im_rms_norm_grad_workspace(n, d) for n in list(range(0, 9000, 7)) + [65536, 1 << 20]]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("i,o,parts", [(1408, 1536, 3), (1536, 2048, 2), (1024, 512, 16), (1024, 1024, 8), (2048, 2304, 1)])
def test_many_rows_parts_of_dw(lib, i, o, parts):
    """The weight gradient of many rows is formed in as many parts as its 128 x 128 tiles leave room
    for, whatever their number: the workspace holds the parts beside dy in 8 bits and its sums."""
    n = 65536
    store = 2 * n * o + n * -(-o // 128) + o * n // 128 + n // 128 * o * 4
    assert lib.im_block_linear_grad_workspace(n, i, o) == store + (parts * o * i * 4 if parts > 1 else 0)
