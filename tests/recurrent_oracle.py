"""Plain 64-bit forms of a recurrent policy's operators (numpy), used only by the tests."""
import numpy as np

U32 = 2.0 ** -24                      # half a step of fp32, relative
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}

# magnitudes of e4m3 by code 0 .. 126
E4M3 = np.array([c / 512.0 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 10) for c in range(127)])
_MIDDLE = (E4M3[1:] + E4M3[:-1]) / 2


def e4m3(v):
    """Codes (bytes) of v rounded to nearest, ties to the even code; |v| <= 464."""
    a = np.abs(v)
    i = np.searchsorted(_MIDDLE, a)
    tie = (i < 126) & (_MIDDLE[np.minimum(i, 125)] == a) & (i % 2 == 1)
    i = np.minimum(i + tie, 126)
    return (i | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def scale_of(top):
    """Scale byte of a block's largest magnitude (float64 of a float32)."""
    if not np.isfinite(top):
        return 255
    for s in range(0, 248):
        if top <= 448.0 * 2.0 ** (s - 127):
            return s
    raise AssertionError(top)


def pack8(x, rows=1):
    """(q, scale) of x (float64 holding float32 values): q [n][padded] bytes."""
    n, d = x.shape
    nb, db = -(-n // rows), -(-d // 128)
    q = np.zeros((n, db * 128), np.uint8)
    scale = np.zeros((nb, db), np.uint8)
    for r in range(nb):
        for c in range(db):
            b = x[r * rows:(r + 1) * rows, c * 128:(c + 1) * 128]
            bad = not np.isfinite(b).all()
            s = 255 if bad else scale_of(np.abs(b).max())
            scale[r, c] = s
            q[r * rows:(r + 1) * rows, c * 128:min(d, (c + 1) * 128)] = \
                0x7F if bad else e4m3(b * 2.0 ** (127 - s))
    return q, scale


def unpack8(q, scale, d, rows=1):
    mag = np.append(E4M3, np.nan)
    v = mag[q[:, :d] & 0x7F] * np.where(q[:, :d] & 0x80, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    s = np.repeat(np.repeat(s, rows, 0)[:q.shape[0]], 128, 1)[:, :d]
    return v * s


def rms_norm(x, residual, gamma, eps):
    h = x if residual is None else x + residual
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    return h, rstd, h * rstd[:, None] * gamma


def rms_norm_grad(dy, h, dh, gamma, rstd):
    u, g = h * rstd[:, None], dy * gamma
    dx = rstd[:, None] * (g - u * (g * u).mean(1, keepdims=True))
    return dx if dh is None else dx + dh, (dy * u).sum(0)


def _sigmoid(g):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))


def scan(gate, x, end, state):
    """(h, c before each step, last c, bounds of an fp32 evaluation's error of h and of c).

    The bounds follow the recursion itself: a step's gate, its complement, the product and the
    sum are off by a few roundings each, 12 in all, relative to a |c| + (1 - a) |x|; a map of
    many steps composed first has the same number of roundings in its products."""
    T, n, d = x.shape
    a, b = _sigmoid(gate)
    h, before = np.zeros_like(x), np.zeros_like(x)
    eh, ebefore = np.zeros_like(x), np.zeros_like(x)
    c, e = state.copy(), np.zeros((n, d))
    for t in range(T):
        before[t], ebefore[t] = c, e
        h[t] = a[t] * c + b[t] * x[t]
        eh[t] = a[t] * e + 12 * U32 * (a[t] * np.abs(c) + b[t] * np.abs(x[t]))
        live = ~end[t][:, None]
        c, e = np.where(live, h[t], 0.0), np.where(live, eh[t], 0.0)
    return h, before, c, eh, ebefore, e


def scan_grad(dh, gate, x, end, before, ebefore, dstate):
    """(dgate, dx, dstate_out, bounds of each), as scan's."""
    T, n, d = x.shape
    a, b = _sigmoid(gate)
    out = [np.zeros_like(x) for _ in range(4)]
    dgate, dx, edgate, edx = out
    D, e = dstate.copy(), np.zeros((n, d))
    for t in range(T - 1, -1, -1):
        live = ~end[t][:, None]
        carry = np.where(live, D, 0.0)
        G, eG = dh[t] + carry, np.where(live, e, 0.0) + 4 * U32 * (np.abs(dh[t]) + np.abs(carry))
        dx[t], edx[t] = b[t] * G, b[t] * (eG + 12 * U32 * np.abs(G))
        diff, ediff = before[t] - x[t], ebefore[t] + 4 * U32 * (np.abs(before[t]) + np.abs(x[t]))
        dgate[t] = a[t] * b[t] * diff * G
        edgate[t] = a[t] * b[t] * (np.abs(diff) * eG + (np.abs(G) + eG) * ediff
                                   + 16 * U32 * np.abs(diff * G))
        D, e = a[t] * G, a[t] * (eG + 12 * U32 * np.abs(G))
    return dgate, dx, D, edgate, edx, e
