"""The operators of a layer of experts, as measured cases.

A policy for many clips has hidden layers whose weights go by the env: rows
(envs or samples) are grouped by expert, normed, and multiplied by their own
expert's weights; the update keeps what the backward pass needs in 8 bits.

  group      rows by expert: offsets and row order from each row's expert
  linear     the grouped product with bias and ReLU
  lgrad      its gradients: input, weights, bias; the input in bf16 or in 8 bits
  norm       layer norm with its row statistics, optionally the 8-bit checkpoint of its input
  ngrad      its gradients, from the input or from its checkpoint
  ckpt       an activation stored in 8 bits and loaded again

Sizes are those of the S15 and S24 humanoids' policies (observations of 226,
361 and 538 values, hidden layers of 1024 and 512, 28 and 69 actions), from one
env to an update's minibatch of 524288 samples.
"""
import torch

own = False

DEV = "cuda"
EPS = 1e-5
BLOCK = 32            # values that share a scale in a checkpoint
MAX_ELEMS = 524288 * 512


def listed():
    return [
        # a player's single env, full precision: latency
        dict(name="norm_f32_1x1024", kind="norm", n=1, d=1024, f32=True, ckpt=False, pad=0),
        # a rollout step of the large batch, its input kept for the update
        dict(name="norm_bf16_65536x1024_ckpt", kind="norm", n=65536, d=1024, f32=False, ckpt=True,
             pad=0),
        # one minibatch of the largest update, from the checkpoint
        dict(name="ngrad_bf16_524288x512_ckpt", kind="ngrad", n=524288, d=512, f32=False, ckpt=True,
             pad=0),
        # observations of the S24 humanoid as they lie, odd rows and width
        dict(name="ngrad_f32_4097x361", kind="ngrad", n=4097, d=361, f32=True, ckpt=False, pad=0),
        # a small batch's observations with training terms kept in 8 bits
        dict(name="ckpt_f32_4096x538", kind="ckpt", n=4096, d=538, f32=True, pad=0),
        # hidden activations of a minibatch
        dict(name="ckpt_bf16_262144x1024", kind="ckpt", n=262144, d=1024, f32=False, pad=0),
        # a few served envs; the whole batch after a reset, clips unevenly drawn
        dict(name="group_64_e8", kind="group", n=64, experts=8, skew=False, drop=False),
        dict(name="group_262144_e64", kind="group", n=262144, experts=64, skew=True, drop=True),
        # served envs through the S24 first layer: a few rows for each expert
        dict(name="linear_64_361x1024_e8", kind="linear", n=64, experts=8, din=361, dout=1024,
             skew=False, order=True, relu=True, pad=7),
        # the large batch through a hidden layer, clips unevenly drawn
        dict(name="linear_65536_1024x1024_e16", kind="linear", n=65536, experts=16, din=1024,
             dout=1024, skew=True, order=True, relu=True, pad=0),
        # its update, the layer's input from the checkpoint
        dict(name="lgrad_65536_1024x512_e16_ckpt", kind="lgrad", n=65536, experts=16, din=1024,
             dout=512, skew=True, order=True, relu=True, ckpt=True, pad=0),
        # a small update on observations as they lie, rows grouped already
        dict(name="lgrad_4095_361x1024_e8", kind="lgrad", n=4095, experts=8, din=361, dout=1024,
             skew=False, order=False, relu=False, ckpt=False, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["group", "linear", "linear", "lgrad", "lgrad", "norm", "ngrad", "ckpt"])
    if kind == "group":
        return dict(kind=kind, n=_log(rng, 1, 262144), experts=_log(rng, 1, 256),
                    skew=rng.random() < 0.5, drop=rng.random() < 0.5)
    if kind in ("linear", "lgrad"):
        din, dout = _log(rng, 28, 1024), _log(rng, 28, 1024)
        c = dict(kind=kind, n=_log(rng, 1, 65536), experts=_log(rng, 1, 32), din=din, dout=dout,
                 skew=rng.random() < 0.5, order=rng.random() < 0.7, relu=rng.random() < 0.5)
        if kind == "lgrad":
            c["ckpt"] = rng.random() < 0.5
            c["n"] = max(1, c["n"] // 2)
        # rows as they lie, or padded to 16 bytes
        c["pad"] = 0 if rng.random() < 0.3 else -din % 8
        return c
    d = _log(rng, 1 if kind == "ckpt" else 28, 4096)
    n = _log(rng, 1, min(262144, MAX_ELEMS // 2 // d))
    c = dict(kind=kind, n=n, d=d, f32=rng.random() < 0.5)
    if kind != "ckpt":
        c["ckpt"] = rng.random() < 0.5
    c["pad"] = rng.choice([0, -d % 8, 3])
    return c


def _blocks(d):
    return -(-d // BLOCK)


def _ckpt_bytes(n, d):
    return n * (d + _blocks(d))


def work(case):
    k, n = case["kind"], case["n"]
    if k == "group":
        return {"bytes": 8 * n + 4 * (case["experts"] + 1), "flops": 0}
    if k in ("linear", "lgrad"):
        e, i, o = case["experts"], case["din"], case["dout"]
        idx = (4 * n if case["order"] else 0) + 4 * (e + 1)
        if k == "linear":
            return {"bytes": 2 * n * (i + o) + 2 * e * o * i + 4 * e * o + idx, "flops": 2 * n * i * o}
        x = _ckpt_bytes(n, i) if case["ckpt"] else 2 * n * i
        return {"bytes": x + 2 * n * (o + i) + 2 * e * o * i + 4 * e * o * (i + 1) + idx,
                "flops": 4 * n * i * o}
    d, s = case["d"], 4 if case["f32"] else 2
    if k == "norm":
        # the checkpoint is written, read and restored
        c = 2 * _ckpt_bytes(n, d) + s * n * d if case["ckpt"] else 0
        return {"bytes": 2 * s * n * d + 8 * n + 8 * d + c, "flops": 8 * n * d}
    if k == "ngrad":
        x = _ckpt_bytes(n, d) if case["ckpt"] else s * n * d
        return {"bytes": x + 2 * s * n * d + 8 * n + 12 * d, "flops": 14 * n * d}
    return {"bytes": 2 * s * n * d + 2 * _ckpt_bytes(n, d), "flops": 4 * n * d}


# ------------------------------------------------------------------- inputs
def _strided(x, pad):
    """x as rows of a wider array."""
    if not pad:
        return x.contiguous()
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _empty(n, d, pad, dtype):
    return torch.zeros((n, d + pad), dtype=dtype, device=DEV)[:, :d]


def _normal(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _experts(case, g):
    """Each row's expert; with skew the k-th has a share of about 1 / (k + 1)."""
    n, e = case["n"], case["experts"]
    u = torch.rand(n, device=DEV, generator=g)
    if case["skew"]:
        share = 1.0 / torch.arange(1, e + 1, device=DEV, dtype=torch.float64)
        edge = (share.cumsum(0) / share.sum()).float()
        k = torch.searchsorted(edge, u).clamp(max=e - 1)
    else:
        k = (u * e).long().clamp(max=e - 1)
    if case.get("drop"):      # envs that are not played now
        k = torch.where(torch.rand(n, device=DEV, generator=g) < 0.05, torch.full_like(k, -1), k)
    return k.to(torch.int32)


def _checkpoint(x):
    """(q, scale) of x: q = round(x / 2^(E - 133)) in blocks of 32, E - 127 the exponent of the
    block's largest magnitude, one more where that would round to 128."""
    n, d = x.shape
    nb = _blocks(d)
    b = torch.zeros((n, nb * BLOCK), device=x.device)
    b[:, :d] = x.float()
    b = b.view(n, nb, BLOCK)
    top = b.abs().amax(2)
    m, e = torch.frexp(top)
    e = e - 1 + (m >= 127.5 / 128).to(e.dtype)
    scale = torch.where(top > 0, (e + 127).clamp(0, 254), torch.zeros_like(e))
    q = torch.round(b / _step(scale)[:, :, None]).clamp(-127, 127)
    return q.to(torch.int8).view(n, -1)[:, :d].contiguous(), scale.to(torch.uint8)


def _step(scale):
    """2^(scale - 133) by its bits (exp2 need not be exact); activations lie far above 2^-120."""
    return ((scale.to(torch.int32).clamp(min=7) - 6) << 23).view(torch.float32)


def _restore(q, scale):
    n, d = q.shape
    return q.float() * _step(scale).repeat_interleave(BLOCK, dim=1)[:, :d]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    k, n = case["kind"], case["n"]
    s = dict(case=case)
    if k == "group":
        s["expert"] = _experts(case, g)
        s["offsets"] = torch.zeros(case["experts"] + 1, dtype=torch.int32, device=DEV)
        s["rows"] = torch.zeros(n, dtype=torch.int32, device=DEV)
        return s
    if k in ("linear", "lgrad"):
        e, i, o, pad = case["experts"], case["din"], case["dout"], case["pad"]
        ex = _experts(case, g)
        if not case["order"]:
            ex = ex.sort().values
        count = torch.bincount(ex.long(), minlength=e)
        s["cap"] = int(count.max())
        s["offsets"] = torch.cat([count.new_zeros(1), count.cumsum(0)]).to(torch.int32)
        s["rows"] = torch.argsort(ex, stable=True).to(torch.int32) if case["order"] else None
        x = _normal(g, n, i)
        if k == "lgrad" and case["relu"]:
            x = x.clamp(min=0)
        s["x"] = _strided(x.bfloat16(), pad)
        w = (_normal(g, e * o, i) * (2.0 / i) ** 0.5).bfloat16()
        s["w"] = _strided(w, pad).unflatten(0, (e, o))
        s["bias"] = 0.1 * _normal(g, e, o)
        if k == "linear":
            s["y"] = torch.zeros((n, o), dtype=torch.bfloat16, device=DEV)
            return s
        s["dy"] = (_normal(g, n, o) * 1e-3).bfloat16()
        s["dx"] = _empty(n, i, pad, torch.bfloat16)
        s["dw"] = torch.zeros((e, o, i), device=DEV)
        s["db"] = torch.zeros((e, o), device=DEV)
        if case["ckpt"]:
            s["q"], s["scale"] = _checkpoint(s.pop("x"))
        return s
    d, pad = case["d"], case["pad"]
    dt = torch.float32 if case["f32"] else torch.bfloat16
    # activations: columns of their own offset and spread
    x = _normal(g, n, d) * (0.5 + torch.rand(d, device=DEV, generator=g)) + 0.5 * _normal(g, d)
    x = _strided(x.to(dt), pad)
    if k == "ckpt":
        s["x"] = x
        s["q"] = torch.zeros((n, d), dtype=torch.int8, device=DEV)
        s["scale"] = torch.zeros((n, _blocks(d)), dtype=torch.uint8, device=DEV)
        s["back"] = _empty(n, d, pad, dt)
        return s
    s["gamma"] = 1.0 + 0.2 * _normal(g, d)
    s["beta"] = 0.1 * _normal(g, d)
    s["mean"] = torch.zeros(n, device=DEV)
    s["rstd"] = torch.zeros(n, device=DEV)
    if k == "norm":
        s["x"] = x
        s["y"] = _empty(n, d, pad, dt)
        if case["ckpt"]:
            s["q"] = torch.zeros((n, d), dtype=torch.int8, device=DEV)
            s["scale"] = torch.zeros((n, _blocks(d)), dtype=torch.uint8, device=DEV)
            s["back"] = torch.zeros((n, d), dtype=dt, device=DEV)
        return s
    xf = x.float()
    s["mean"] = xf.mean(1)
    s["rstd"] = 1.0 / torch.sqrt((xf - s["mean"][:, None]).square().mean(1) + EPS)
    del xf
    s["dy"] = _strided((_normal(g, n, d) * 1e-3).to(dt), pad)
    s["dx"] = _empty(n, d, pad, dt)
    s["dgamma"] = torch.zeros(d, device=DEV)
    s["dbeta"] = torch.zeros(d, device=DEV)
    if case["ckpt"]:
        s["q"], s["scale"] = _checkpoint(x)
    else:
        s["x"] = x
    return s


# --------------------------------------------------------------- plain forms
def _plain_group(s):
    e = s["case"]["experts"]
    k = s["expert"]
    k = torch.where((k >= 0) & (k < e), k, torch.full_like(k, e))
    sorted_, rows = torch.sort(k, stable=True)
    offsets = torch.searchsorted(sorted_, torch.arange(e + 1, dtype=k.dtype, device=k.device))
    return [offsets.to(torch.int32), rows.to(torch.int32)]


def _places(s, n):
    """For each expert its rows, padded to the largest group: (row index, valid, target)."""
    off = s["offsets"].long()
    at = off[:-1, None] + torch.arange(s["cap"], device=off.device)
    valid = at < off[1:, None]
    at = at.clamp(max=n - 1)
    row = s["rows"].long()[at] if s["rows"] is not None else at
    return row, valid[:, :, None], torch.where(valid, row, torch.full_like(row, n)).view(-1)


def _scatter(v, target, n):
    out = torch.zeros((n + 1, v.shape[-1]), device=v.device)
    out[target] = v.reshape(-1, v.shape[-1])
    return out[:n]


def _plain_linear(s):
    n = s["case"]["n"]
    row, valid, target = _places(s, n)
    x = s["x"].float()[row] * valid
    y = torch.bmm(x, s["w"].float().transpose(1, 2)) + s["bias"][:, None, :]
    if s["case"]["relu"]:
        y = y.clamp(min=0)
    return _scatter(y, target, n).bfloat16()


def _plain_lgrad(s):
    n = s["case"]["n"]
    row, valid, target = _places(s, n)
    x = _restore(s["q"], s["scale"]) if s["case"]["ckpt"] else s["x"].float()
    x = x[row] * valid
    dy = s["dy"].float()[row] * valid
    dx = torch.bmm(dy, s["w"].float())
    if s["case"]["relu"]:
        dx = dx * (x > 0)
    dw = torch.bmm(dy.transpose(1, 2), x)
    return [_scatter(dx, target, n).bfloat16(), dw, dy.sum(1)]


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt(c.square().mean(1) + EPS)
    y = (c * rstd[:, None] * s["gamma"] + s["beta"]).to(s["x"].dtype)
    out = [y, mean, rstd]
    if s["case"]["ckpt"]:
        out.append(_restore(*_checkpoint(s["x"])).to(s["x"].dtype))
    return out


def _plain_ngrad(s):
    x = _restore(s["q"], s["scale"]) if s["case"]["ckpt"] else s["x"].float()
    h = (x - s["mean"][:, None]) * s["rstd"][:, None]
    dy = s["dy"].float()
    g = dy * s["gamma"]
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return [dx.to(s["dy"].dtype), (dy * h).sum(0), dy.sum(0)]


def _plain_ckpt(s):
    return _restore(*_checkpoint(s["x"])).to(s["x"].dtype)


# ------------------------------------------------------- the framework's calls
def _run_own(s):
    from paper_2609_09821_amd import binding as im

    c = s["case"]
    k, n = c["kind"], c["n"]
    ckpt = im.Checkpoint(s["q"], s["scale"]) if "q" in s else None
    if k == "group":
        if "ws" not in s:
            s["ws"] = im.group_rows_workspace(n, c["experts"])
        im.group_rows(s["expert"], s["offsets"], s["rows"], s["ws"])
        return [s["offsets"], s["rows"]]
    if k == "linear":
        im.expert_linear(s["x"], s["w"], s["bias"], s["offsets"], s["rows"], s["y"], relu=c["relu"])
        return s["y"]
    if k == "lgrad":
        if "ws" not in s:
            s["ws"] = im.expert_linear_grad_workspace(n, c["experts"], c["din"], c["dout"])
        im.expert_linear_grad(s["dy"], ckpt if c["ckpt"] else s["x"], s["w"], s["offsets"],
                              s["rows"], s["dx"], s["dw"], s["db"], relu_x=c["relu"],
                              workspace=s["ws"])
        return [s["dx"], s["dw"], s["db"]]
    if k == "norm":
        im.layer_norm(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], eps=EPS,
                      checkpoint=ckpt)
        if ckpt is None:
            return [s["y"], s["mean"], s["rstd"]]
        im.checkpoint_load(ckpt, s["back"])
        return [s["y"], s["mean"], s["rstd"], s["back"]]
    if k == "ngrad":
        if "ws" not in s:
            s["ws"] = im.layer_norm_grad_workspace(n, c["d"])
        im.layer_norm_grad(s["dy"], ckpt if c["ckpt"] else s["x"], s["gamma"], s["mean"], s["rstd"],
                           s["dx"], s["dgamma"], s["dbeta"], workspace=s["ws"])
        return [s["dx"], s["dgamma"], s["dbeta"]]
    im.checkpoint_store(s["x"], ckpt)
    im.checkpoint_load(ckpt, s["back"])
    return s["back"]


def run(state):
    if own:
        return _run_own(state)
    return {"group": _plain_group, "linear": _plain_linear, "lgrad": _plain_lgrad,
            "norm": _plain_norm, "ngrad": _plain_ngrad, "ckpt": _plain_ckpt}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ in 64 bits
def _power(e):
    """2^e in float64, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_restored(x):
    """The checkpoint's values: in each block of columns the smallest power of two as step
    that takes the largest magnitude to at most 127."""
    x = x.double()
    out = torch.empty_like(x)
    for c0 in range(0, x.shape[1], BLOCK):
        b = x[:, c0:c0 + BLOCK]
        top = b.abs().amax(1, keepdim=True)
        # a first exponent that is too small, then up to where the magnitude rounds to 127 at most
        e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 8
        for _ in range(4):
            e = torch.where(torch.round(top / _power(e)) > 127, e + 1, e)
        out[:, c0:c0 + BLOCK] = torch.round(b / _power(e)) * _power(e)
    return out


def _exact_stored(q, scale):
    v = q.double()
    for b in range(scale.shape[1]):
        v[:, b * BLOCK:(b + 1) * BLOCK] *= _power(scale[:, b:b + 1].long() - 133)
    return v


def exact(case, seed):
    k = case["kind"]
    if k == "group":
        return None
    s = prepare(case, seed)
    if k in ("linear", "lgrad"):
        n, e = case["n"], case["experts"]
        off = s["offsets"].tolist()
        place = s["rows"].long() if s["rows"] is not None else torch.arange(n, device=DEV)
        if k == "linear":
            y = torch.zeros((n, case["dout"]), dtype=torch.float64, device=DEV)
            for j in range(e):
                r = place[off[j]:off[j + 1]]
                v = s["x"][r].double() @ s["w"][j].double().t() + s["bias"][j].double()
                y[r] = torch.maximum(v, torch.zeros_like(v)) if case["relu"] else v
            return y
        x = _exact_stored(s["q"], s["scale"]) if case["ckpt"] else s["x"].double()
        dy = s["dy"].double()
        dx = torch.zeros((n, case["din"]), dtype=torch.float64, device=DEV)
        dw = torch.zeros((e, case["dout"], case["din"]), dtype=torch.float64, device=DEV)
        db = torch.zeros((e, case["dout"]), dtype=torch.float64, device=DEV)
        for j in range(e):
            r = place[off[j]:off[j + 1]]
            dx[r] = dy[r] @ s["w"][j].double()
            dw[j] = dy[r].t() @ x[r]
            db[j] = dy[r].sum(0)
        if case["relu"]:
            dx[~(x > 0)] = 0.0
        return [dx, dw, db]
    if k == "ckpt":
        return _exact_restored(s["x"])
    gamma = s["gamma"].double()
    if k == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = (var + EPS) ** -0.5
        y = (x - mean[:, None]) * rstd[:, None] * gamma + s["beta"].double()
        return [y, mean, rstd] + ([_exact_restored(s["x"])] if case["ckpt"] else [])
    x = _exact_stored(s["q"], s["scale"]) if case["ckpt"] else s["x"].double()
    mean, rstd = s["mean"].double()[:, None], s["rstd"].double()[:, None]
    h, dy = (x - mean) * rstd, s["dy"].double()
    g = dy * gamma
    d = case["d"]
    dx = g - (g.sum(1, keepdim=True) + h * (g * h).sum(1, keepdim=True)) / d
    return [dx * rstd, (dy * h).sum(0), dy.sum(0)]
