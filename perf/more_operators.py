"""The operators of a recurrent policy in 8 bits, as measured cases.

A policy that remembers has blocks of: a root-mean-square norm of the residual stream, products
in 8-bit floating point, and a gated linear recurrence over the rollout's steps, whose state is
cleared where an episode ends.

  norm     root-mean-square norm, optionally of a sum with the residual, its output optionally
           in 8 bits
  ngrad    its gradients
  linear   the product with weights in 8 bits, bias and ReLU; the operands stored in 8 bits
           before or in the same pass, the output in 32, 16 or 8 bits
  lgrad    its gradients: input, weights, bias
  scan     the recurrence over T steps of n envs from a state
  sgrad    its gradients

8 bits are e4m3 values in blocks that share a power of two: 128 consecutive values of a row, for
weights 128 x 128.  Sizes are those of the S15 and S24 humanoids' policies (observations of 226,
361 and 538 values, hidden layers of 1024 and 512) and of rollouts of 32 steps, from one env to an
update's minibatch of 524288 samples, and single long episodes.
"""
import torch

own = False

DEV = "cuda"
EPS = 1e-6
BLOCK = 128           # values that share a scale
KEEP = 16             # steps between the states that a scan keeps for its gradient
MAX_ELEMS = 65536 * 1024


def listed():
    return [
        # a player's single env, full precision: latency
        dict(name="norm_f32_1x1024", kind="norm", n=1, d=1024, f32=True, res=False, y=True, y8=False,
             pad=0),
        # a rollout step of the large batch between two blocks: the residual's sum, 8 bits out
        dict(name="norm_bf16_65536x1024_res_8bit", kind="norm", n=65536, d=1024, f32=False, res=True,
             y=False, y8=True, pad=0),
        # one minibatch of the largest update, the residual's gradient added
        dict(name="ngrad_bf16_524288x512_res", kind="ngrad", n=524288, d=512, f32=False, res=True,
             pad=0),
        # observations of the S24 humanoid as they lie, odd rows and width
        dict(name="ngrad_f32_4097x361", kind="ngrad", n=4097, d=361, f32=True, res=False, pad=0),
        # a served env's observation through the S24 first layer
        dict(name="linear_1_361x1024_store", kind="linear", n=1, din=361, dout=1024, relu=True,
             fresh="x", out="bf16", f32=True, pad=0),
        # the large batch through a hidden layer, in 8 bits already
        dict(name="linear_65536_1024x1024", kind="linear", n=65536, din=1024, dout=1024, relu=True,
             fresh="", out="bf16", f32=False, pad=0),
        # its update
        dict(name="lgrad_65536_1024x512_relu", kind="lgrad", n=65536, din=1024, dout=512, relu=True,
             f32=False, pad=0),
        # a small update on observations, odd rows and width
        dict(name="lgrad_4095_361x1024", kind="lgrad", n=4095, din=361, dout=1024, relu=False,
             f32=False, pad=0),
        # one step of a few served envs
        dict(name="scan_f32_1x64x512", kind="scan", t=1, n=64, d=512, f32=True, done=True, state=True,
             pad=0),
        # a rollout of a large batch, gates and values the two halves of one product's rows
        dict(name="scan_bf16_32x16384x256", kind="scan", t=32, n=16384, d=256, f32=False, done=True,
             state=True, pad=256),
        # its update
        dict(name="sgrad_bf16_32x16384x256", kind="sgrad", t=32, n=16384, d=256, f32=False, done=True,
             state=True, pad=256),
        # two long episodes, odd width
        dict(name="sgrad_f32_16383x2x361", kind="sgrad", t=16383, n=2, d=361, f32=True, done=True,
             state=False, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["norm", "ngrad", "linear", "linear", "lgrad", "scan", "scan", "sgrad"])
    f32 = rng.random() < 0.5
    if kind in ("norm", "ngrad"):
        d = _log(rng, 16, 4096)
        c = dict(kind=kind, n=_log(rng, 1, min(262144, MAX_ELEMS // 2 // d)), d=d, f32=f32,
                 res=rng.random() < 0.5, pad=rng.choice([0, -d % 8, 3]))
        if kind == "norm":
            c["y8"] = rng.random() < 0.5
            c["y"] = not c["y8"] or rng.random() < 0.5
        return c
    if kind in ("linear", "lgrad"):
        c = dict(kind=kind, n=_log(rng, 1, 65536), din=_log(rng, 16, 1024),
                 dout=_log(rng, 16, 1024), relu=rng.random() < 0.5, f32=f32)
        c["pad"] = rng.choice([0, 3])
        if kind == "linear":
            c["fresh"] = rng.choice(["", "", "x", "xw"])
            c["out"] = rng.choice(["bf16", "f32", "8"])
        else:
            c["n"] = max(1, c["n"] // 2)
        return c
    t, d = _log(rng, 1, 16384), _log(rng, 1, 1024)
    n = _log(rng, 1, max(1, min(65536, MAX_ELEMS // 2 // (t * d))))
    return dict(kind=kind, t=t, n=n, d=d, f32=f32, done=rng.random() < 0.7,
                state=rng.random() < 0.5, pad=rng.choice([0, -d % 8, d]))


def _blocks(d):
    return -(-d // BLOCK)


def work(case):
    k, n, s = case["kind"], case["n"], 4 if case["f32"] else 2
    if k == "norm":
        d = case["d"]
        b = s * n * d + 4 * n + 4 * d
        if case["res"]:
            b += 2 * s * n * d
        if case["y"]:
            b += s * n * d
        if case["y8"]:      # written, read and restored as bf16
            b += 2 * n * (d + _blocks(d)) + 2 * n * d
        return {"bytes": b, "flops": 6 * n * d}
    if k == "ngrad":
        d = case["d"]
        return {"bytes": (4 if case["res"] else 3) * s * n * d + 4 * n + 8 * d, "flops": 10 * n * d}
    if k == "linear":
        i, o = case["din"], case["dout"]
        x8, w8 = n * (i + _blocks(i)), o * i + _blocks(o) * _blocks(i)
        b = x8 + w8 + 4 * o
        if "x" in case["fresh"]:
            b += s * n * i + x8
        if "w" in case["fresh"]:
            b += 4 * o * i + w8
        b += {"bf16": 2 * n * o, "f32": 4 * n * o, "8": 2 * n * (o + _blocks(o)) + 2 * n * o}[case["out"]]
        return {"bytes": b, "flops": 2 * n * i * o}
    if k == "lgrad":
        i, o = case["din"], case["dout"]
        b = (2 if case["relu"] else 1) * s * n * o + i * n + i * _blocks(n) + i * o + _blocks(i) * _blocks(o)
        return {"bytes": b + s * n * i + 4 * o * i + 4 * o, "flops": 4 * n * i * o}
    t, d = case["t"], case["d"]
    m = t * n * d
    flags = 2 * t * n if case["done"] else 0
    if k == "scan":
        return {"bytes": 3 * s * m + 4 * n * d * (2 if case["state"] else 1) + flags, "flops": 8 * m}
    kept = 4 * n * d * -(-t // KEEP)
    return {"bytes": 5 * s * m + kept + 4 * n * d * (2 if case["state"] else 1) + flags, "flops": 20 * m}


# ------------------------------------------------------------------- inputs
def _strided(x, pad):
    """x as rows of a wider array."""
    if not pad:
        return x.contiguous()
    wide = torch.zeros((*x.shape[:-1], x.shape[-1] + pad), dtype=x.dtype, device=x.device)
    wide[..., :x.shape[-1]] = x
    return wide[..., :x.shape[-1]]


def _empty(shape, pad, dtype):
    return torch.zeros((*shape[:-1], shape[-1] + pad), dtype=dtype, device=DEV)[..., :shape[-1]]


def _normal(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _power(e):
    """2^e for whole e in -126..127, by its bits (exp2 need not be exact)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _pack8(x, rows=1):
    """(q, scale) of x: q e4m3 in rows padded with zeros to whole blocks, value = q 2^(scale - 127);
    the scale is the smallest that takes a block's largest magnitude to at most 448."""
    n, d = x.shape
    nb, db = -(-n // rows), _blocks(d)
    v = torch.zeros((nb * rows, db * BLOCK), device=x.device)
    v[:n, :d] = x.float()
    v = v.view(nb, rows, db, BLOCK)
    m, e = torch.frexp(v.abs().amax((1, 3)))
    # the largest magnitude is m 2^e with m in [0.5, 1); 448 is 0.875 2^9
    scale = torch.where(m > 0, (e - 9 + (m > 0.875).to(e.dtype) + 127).clamp(min=0), torch.zeros_like(e))
    q = (v * _power(127 - scale)[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(nb * rows, -1)[:n].contiguous(), scale.to(torch.uint8)


def _unpack8(q, scale, d, rows=1):
    """The values, exact in 32 bits and in bf16 (scales of activations are far above 2^-126)."""
    s = _power(scale.to(torch.int32) - 127)
    s = s.repeat_interleave(rows, dim=0)[:q.shape[0]].repeat_interleave(BLOCK, dim=1)
    return (q.float() * s)[:, :d]


def _empty8(n, d, rows=1):
    return (torch.zeros((n, _blocks(d) * BLOCK), dtype=torch.float8_e4m3fn, device=DEV),
            torch.zeros((-(-n // rows), _blocks(d)), dtype=torch.uint8, device=DEV))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    k, n, pad = case["kind"], case["n"], case["pad"]
    dt = torch.float32 if case["f32"] else torch.bfloat16
    s = dict(case=case)
    if k in ("norm", "ngrad"):
        d = case["d"]
        # activations: columns of their own spread
        x = _normal(g, n, d) * (0.5 + torch.rand(d, device=DEV, generator=g))
        s["gamma"] = 1.0 + 0.2 * _normal(g, d)
        s["rstd"] = torch.zeros(n, device=DEV)
        s["x"] = _strided(x.to(dt), pad)
        if k == "norm":
            if case["res"]:
                s["res"] = _strided((2.0 * _normal(g, n, d)).to(dt), pad)
                s["h"] = _empty((n, d), pad, dt)
            if case["y"]:
                s["y"] = _empty((n, d), pad, dt)
            if case["y8"]:
                s["q"], s["scale"] = _empty8(n, d)
                s["back"] = torch.zeros((n, d), dtype=torch.bfloat16, device=DEV)
            return s
        s["rstd"] = 1.0 / torch.sqrt(s["x"].float().square().mean(1) + EPS)
        s["dy"] = _strided((_normal(g, n, d) * 1e-3).to(dt), pad)
        if case["res"]:
            s["dh"] = _strided((_normal(g, n, d) * 1e-3).to(dt), pad)
        s["dx"] = _empty((n, d), pad, dt)
        s["dgamma"] = torch.zeros(d, device=DEV)
        return s
    if k in ("linear", "lgrad"):
        i, o = case["din"], case["dout"]
        x = _normal(g, n, i) * (0.5 + torch.rand(i, device=DEV, generator=g))
        w = _normal(g, o, i) * (2.0 / i) ** 0.5
        if k == "linear":
            s["bias"] = 0.1 * _normal(g, o)
            if "x" in case["fresh"]:
                s["x"] = _strided(x.to(dt), pad)
                s["xq"], s["xs"] = _empty8(n, i)
            else:
                s["xq"], s["xs"] = _pack8(x)
            if "w" in case["fresh"]:
                s["w"] = w
                s["wq"], s["ws"] = _empty8(o, i, BLOCK)
            else:
                s["wq"], s["ws"] = _pack8(w, BLOCK)
            if case["out"] == "8":
                s["q"], s["scale"] = _empty8(n, o)
                s["back"] = torch.zeros((n, o), dtype=torch.bfloat16, device=DEV)
            else:
                s["y"] = _empty((n, o), pad, torch.float32 if case["out"] == "f32" else torch.bfloat16)
            return s
        s["xq"], s["xs"] = _pack8(x.t())
        s["wq"], s["ws"] = _pack8(w.t(), BLOCK)
        s["dy"] = _strided((_normal(g, n, o) * 1e-3).to(dt), pad)
        if case["relu"]:
            s["y"] = _strided(_normal(g, n, o).clamp(min=0).to(dt), pad)
        s["dx"] = _empty((n, i), pad, dt)
        s["dw"] = torch.zeros((o, i), device=DEV)
        s["db"] = torch.zeros(o, device=DEV)
        return s
    t, d = case["t"], case["d"]
    # gates that remember for some ten steps, as the first of a product's columns and the values
    # after them where the rows are twice as wide
    s["gate"] = _strided((2.0 + 1.5 * _normal(g, t, n, d)).to(dt), pad)
    s["x"] = _strided(_normal(g, t, n, d).to(dt), pad)
    s["terminated"] = s["truncated"] = None
    if case["done"]:
        u = torch.rand((2, t, n), device=DEV, generator=g)
        s["terminated"], s["truncated"] = (u < 0.02).to(torch.uint8)
    s["state"] = _normal(g, n, d) if case["state"] else None
    if k == "scan":
        s["h"] = _empty((t, n, d), 0, dt)
        s["state_out"] = torch.zeros((n, d), device=DEV)
        return s
    s["dh"] = _strided((_normal(g, t, n, d) * 1e-3).to(dt), pad)
    s["dstate"] = _normal(g, n, d) * 1e-3 if case["state"] else None
    s["keep"] = torch.zeros((-(-t // KEEP), n, d), device=DEV)
    if case["state"]:
        s["keep"][0] = s["state"]
    last = (s["keep"].shape[0] - 1) * KEEP
    if last:
        h = _recur(*_terms(s["gate"][:last], s["x"][:last], _live(s, last), s["keep"][0]))
        s["keep"][1:] = (h * _live(s, last))[KEEP - 1::KEEP]
    s["dgate"], s["dx"] = _empty((t, n, d), 0, dt), _empty((t, n, d), 0, dt)
    s["dstate_out"] = torch.zeros((n, d), device=DEV)
    return s


# --------------------------------------------------------------- plain forms
def _plain_norm(s):
    c = s["case"]
    h = s["x"].float()
    if c["res"]:
        h = h + s["res"].float()
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + EPS)
    y = h * rstd[:, None] * s["gamma"]
    out = [rstd]
    if c["res"]:
        out.append(h.to(s["x"].dtype))
    if c["y"]:
        out.append(y.to(s["x"].dtype))
    if c["y8"]:
        out.append(_unpack8(*_pack8(y), c["d"]).bfloat16())
    return out


def _plain_ngrad(s):
    rstd = s["rstd"][:, None]
    u = s["x"].float() * rstd
    dy = s["dy"].float()
    g = dy * s["gamma"]
    dx = rstd * (g - u * (g * u).mean(1, keepdim=True))
    if s["case"]["res"]:
        dx = dx + s["dh"].float()
    return [dx.to(s["dy"].dtype), (dy * u).sum(0)]


def _plain_linear(s):
    c = s["case"]
    i, o = c["din"], c["dout"]
    xq, xs = _pack8(s["x"]) if "x" in s else (s["xq"], s["xs"])
    wq, ws = _pack8(s["w"], BLOCK) if "w" in s else (s["wq"], s["ws"])
    y = _unpack8(xq, xs, i) @ _unpack8(wq, ws, i, BLOCK).t() + s["bias"]
    if c["relu"]:
        y = y.clamp(min=0)
    if c["out"] == "8":
        return _unpack8(*_pack8(y), o).bfloat16()
    return y.to(s["y"].dtype)


def _plain_lgrad(s):
    c = s["case"]
    n, o = c["n"], c["dout"]
    dy = s["dy"].float()
    if c["relu"]:
        dy = dy * (s["y"] > 0)
    dx = _unpack8(*_pack8(dy), o) @ _unpack8(s["wq"], s["ws"], o, BLOCK).t()
    dw = _unpack8(*_pack8(dy.t()), n) @ _unpack8(s["xq"], s["xs"], n).t()
    return [dx.to(s["dy"].dtype), dw, dy.sum(0)]


def _live(s, t):
    """1 where the state passes on from a step, 0 where the episode ends with it; [t][n][1]."""
    if s["terminated"] is None:
        return torch.ones((t, s["gate"].shape[1], 1), device=DEV)
    return ((s["terminated"][:t] | s["truncated"][:t]) == 0).float()[:, :, None]


def _terms(gate, x, live, state):
    """a and b of h_t = a_t h_(t-1) + b_t from h_(-1) = 0."""
    gate = gate.float()
    a = 1.0 / (1.0 + torch.exp(-gate))
    b = x.float() / (1.0 + torch.exp(gate))
    b[0] += a[0] * state
    a[1:] *= live[:-1]
    return a, b


def _recur(a, b):
    """All h by doubling: steps that know the last s take in those before them."""
    s = 1
    while s < a.shape[0]:
        b = torch.cat([b[:s], torch.addcmul(b[s:], a[s:], b[:-s])])
        a = torch.cat([a[:s], a[s:] * a[:-s]])
        s *= 2
    return b


def _plain_scan(s):
    t, n, d = s["x"].shape
    live = _live(s, t)
    state = torch.zeros((n, d), device=DEV) if s["state"] is None else s["state"]
    h = _recur(*_terms(s["gate"], s["x"], live, state))
    return [h.to(s["x"].dtype), h[-1] * live[-1]]


def _plain_sgrad(s):
    t = s["case"]["t"]
    live = _live(s, t)
    h = _recur(*_terms(s["gate"], s["x"], live, s["keep"][0]))
    before = torch.cat([s["keep"][:1], (h * live)[:-1]])
    del h
    gate = s["gate"].float()
    a, b = 1.0 / (1.0 + torch.exp(-gate)), 1.0 / (1.0 + torch.exp(gate))
    # G_t = dh_t + live_t a_(t+1) G_(t+1), as a recurrence over the steps backwards
    back, dh = torch.zeros_like(a), s["dh"].float().flip(0)
    back[1:] = (a[1:] * live[:-1]).flip(0)
    if s["dstate"] is not None:
        dh[0] += live[-1] * s["dstate"]
    G = _recur(back, dh).flip(0)
    dt = s["dh"].dtype
    return [(a * b * (before - s["x"].float()) * G).to(dt), (b * G).to(dt), a[0] * G[0]]


# ------------------------------------------------------- the framework's calls
def _run_own(s):
    from paper_2609_09821_amd import binding as im

    c = s["case"]
    k, n = c["kind"], c["n"]
    if k == "norm":
        y8 = im.Block8(s["q"], s["scale"], c["d"]) if c["y8"] else None
        im.rms_norm(s["x"], s["gamma"], s.get("y"), s["rstd"], eps=EPS, residual=s.get("res"),
                    h=s.get("h"), y8=y8)
        if c["y8"]:
            im.block8_load(y8, s["back"])
        return [s[v] for v in ("rstd", "h", "y", "back") if v in s]
    if k == "ngrad":
        if "work" not in s:
            s["work"] = im.rms_norm_grad_workspace(n, c["d"])
        im.rms_norm_grad(s["dy"], s["x"], s["gamma"], s["rstd"], s["dx"], s["dgamma"], dh=s.get("dh"),
                         workspace=s["work"])
        return [s["dx"], s["dgamma"]]
    if k == "linear":
        x8 = im.Block8(s["xq"], s["xs"], c["din"])
        w8 = im.Block8(s["wq"], s["ws"], c["din"], rows=BLOCK)
        if "x" in s:
            im.block8_store(s["x"], x8)
        if "w" in s:
            im.block8_store(s["w"], w8)
        y8 = im.Block8(s["q"], s["scale"], c["dout"]) if c["out"] == "8" else None
        im.linear8(x8, w8, s["bias"], s.get("y"), y8=y8, relu=c["relu"])
        if y8 is None:
            return s["y"]
        im.block8_load(y8, s["back"])
        return s["back"]
    if k == "lgrad":
        if "work" not in s:
            s["work"] = im.linear8_grad_workspace(n, c["din"], c["dout"])
        im.linear8_grad(s["dy"], im.Block8(s["xq"], s["xs"], n),
                        im.Block8(s["wq"], s["ws"], c["dout"], rows=BLOCK), s["dx"], s["dw"], s["db"],
                        y=s.get("y"), workspace=s["work"])
        return [s["dx"], s["dw"], s["db"]]
    if "work" not in s:
        s["work"] = im.gated_scan_workspace(c["t"], n, c["d"])
    if k == "scan":
        im.gated_scan(s["gate"], s["x"], s["h"], s["state"], s["state_out"], terminated=s["terminated"],
                      truncated=s["truncated"], workspace=s["work"])
        return [s["h"], s["state_out"]]
    im.gated_scan_grad(s["dh"], s["gate"], s["x"], s["keep"], s["dgate"], s["dx"], s["dstate"],
                       s["dstate_out"], terminated=s["terminated"], truncated=s["truncated"],
                       workspace=s["work"])
    return [s["dgate"], s["dx"], s["dstate_out"]]


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "ngrad": _plain_ngrad, "linear": _plain_linear, "lgrad": _plain_lgrad,
            "scan": _plain_scan, "sgrad": _plain_sgrad}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ in 64 bits
def _power64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_rounded(v, rows=1):
    """The values that 8 bits hold of v, by a table of the magnitudes 0 .. 448."""
    n, d = v.shape
    code = torch.arange(127, device=v.device)
    table = torch.where(code < 8, code.double() / 512, (8 + code % 8) * _power64(code // 8 - 10))
    middle = (table[1:] + table[:-1]) / 2
    out = torch.empty_like(v, dtype=torch.float64)
    for r0 in range(0, n, rows if rows > 1 else n):
        for c0 in range(0, d, BLOCK):
            b = v[r0:r0 + (rows if rows > 1 else n), c0:c0 + BLOCK].double()
            top = b.abs().amax() if rows > 1 else b.abs().amax(1, keepdim=True)
            # a first exponent that is too small, then up to where the magnitude fits
            e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 11
            for _ in range(5):
                e = torch.where(top / _power64(e) > 448, e + 1, e)
            u = (b / _power64(e)).abs()
            i = torch.searchsorted(middle, u)
            tie = (i < 126) & (middle[i.clamp(max=125)] == u) & (i % 2 == 1)
            out[r0:r0 + b.shape[0], c0:c0 + BLOCK] = table[(i + tie.long()).clamp(max=126)] * torch.sign(b) * _power64(e)
    return out


def _exact_stored(q, scale, d, rows=1):
    v = q[:, :d].double()
    s = _power64(scale.long() - 127)
    for r in range(s.shape[1]):
        v[:, r * BLOCK:(r + 1) * BLOCK] *= s[:, r:r + 1].repeat_interleave(rows, 0)[:v.shape[0]]
    return v


def exact(case, seed):
    s = prepare(case, seed)
    k, n = case["kind"], case["n"]
    if k == "norm":
        h = s["x"].double()
        if case["res"]:
            h += s["res"].double()
        rstd = ((h * h).sum(1) / case["d"] + EPS) ** -0.5
        y = rstd[:, None] * h * s["gamma"].double()
        return [rstd] + ([h] if case["res"] else []) + ([y] if case["y"] else []) + (
            [_exact_rounded(y)] if case["y8"] else [])
    if k == "ngrad":
        # y_j = gamma_j h_j r with r = rstd, and dr / dh_j = -h_j r^3 / d
        h, r, dy = s["x"].double(), s["rstd"].double()[:, None], s["dy"].double()
        through = (dy * s["gamma"].double() * h).sum(1, keepdim=True)
        dx = r * dy * s["gamma"].double() - h * r ** 3 * through / case["d"]
        if case["res"]:
            dx += s["dh"].double()
        return [dx, (dy * h * r).sum(0)]
    if k == "linear":
        i = case["din"]
        x = _exact_rounded(s["x"]) if "x" in s else _exact_stored(s["xq"], s["xs"], i)
        w = _exact_rounded(s["w"], BLOCK) if "w" in s else _exact_stored(s["wq"], s["ws"], i, BLOCK)
        y = torch.addmm(s["bias"].double(), x, w.t())
        if case["relu"]:
            y = torch.maximum(y, torch.zeros_like(y))
        return _exact_rounded(y) if case["out"] == "8" else y
    if k == "lgrad":
        dy = s["dy"].double()
        if case["relu"]:
            dy[~(s["y"] > 0)] = 0.0
        dx = _exact_rounded(dy) @ _exact_stored(s["wq"], s["ws"], case["dout"], BLOCK).t()
        dw = _exact_rounded(dy.t().contiguous()) @ _exact_stored(s["xq"], s["xs"], n).t()
        return [dx, dw, dy.sum(0)]
    t, d = case["t"], case["d"]
    if case["done"]:
        end = (s["terminated"] != 0) | (s["truncated"] != 0)
    else:
        end = torch.zeros((t, n), dtype=torch.bool, device=DEV)
    stop = end[:, :, None]
    c = torch.zeros((n, d), dtype=torch.float64, device=DEV)
    if s["state"] is not None:
        c += s["state"]
    if k == "scan":
        h = torch.zeros((t, n, d), dtype=torch.float64, device=DEV)
        for j in range(t):
            a = torch.sigmoid(s["gate"][j].double())
            h[j] = a * c + (1 - a) * s["x"][j].double()
            c = torch.where(stop[j], 0.0, h[j])
        return [h, c]
    before = torch.zeros((t, n, d), dtype=torch.float64, device=DEV)
    for j in range(t):
        before[j] = c
        a = torch.sigmoid(s["gate"][j].double())
        c = torch.where(stop[j], 0.0, a * c + (1 - a) * s["x"][j].double())
    dgate, dx = torch.zeros_like(before), torch.zeros_like(before)
    # the gradient of the state that a step passes on
    dc = torch.zeros((n, d), dtype=torch.float64, device=DEV)
    if s["dstate"] is not None:
        dc += s["dstate"]
    for j in range(t - 1, -1, -1):
        G = s["dh"][j].double() + torch.where(stop[j], 0.0, dc)
        a = torch.sigmoid(s["gate"][j].double())
        dgate[j] = G * (before[j] - s["x"][j].double()) * a * (1 - a)
        dx[j] = G * (1 - a)
        dc = G * a
    return [dgate, dx, dc]
