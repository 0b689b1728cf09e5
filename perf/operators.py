"""What is measured of the operators around byte checkpoints: activations held in 8 bits between the
forward and the backward pass, and the layers that read them there.

Operators (`op` of a case):
  roundtrip    an activation is stored as a byte checkpoint and restored: x -> x'
  linear_grad  weight (and bias) gradient of a linear layer whose input is held as a byte checkpoint
  norm         group norm with an activation, channels last, nothing saved (inference)
  norm_train   the same with its input saved as a byte checkpoint, then its backward pass from the codes

A byte checkpoint of x[rows, cols] is one buffer of bytes: codes [rows][pitch] with pitch = cols rounded up to
a multiple of 16 (the padding is zero), then one exponent byte e + 127 for every group of `group`
consecutive columns, [rows][ceil(cols / group)], then zeros up to a multiple of 16.  With amax the largest
finite magnitude of a group, e is the exponent for which amax * 2^-e lies in [64, 128) and rounds to at most
127 ("int8"), or lies in [224, 448] ("e4m3"); a code is x * 2^-e rounded to nearest even; x' = code * 2^e.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"bfloat16": torch.bfloat16, "float16": torch.float16, "float32": torch.float32}


def _bytes(dtype: str) -> int:
    return 4 if dtype == "float32" else 2


def _pitch(cols: int) -> int:
    return (cols + 15) // 16 * 16


def _held(case, rows, cols) -> int:
    """Bytes of a checkpoint that carry information."""
    return rows * cols + rows * -(-cols // case["group"])


# --- cases --------------------------------------------------------------------------------------------
def _roundtrip(rows, cols, dtype, fmt, group):
    return {"op": "roundtrip", "rows": rows, "cols": cols, "dtype": dtype, "fmt": fmt, "group": group}


def _linear(rows, cols, outs, dtype, fmt, group, bias):
    return {"op": "linear_grad", "rows": rows, "cols": cols, "outs": outs, "dtype": dtype, "fmt": fmt,
            "group": group, "bias": bias}


def _norm(batch, spatial, channels, groups, act, dtype):
    return {"op": "norm", "batch": batch, "spatial": spatial, "channels": channels, "groups": groups, "act": act,
            "dtype": dtype}


def _train(batch, spatial, channels, groups, act, dtype, fmt, group):
    return {**_norm(batch, spatial, channels, groups, act, dtype), "op": "norm_train", "fmt": fmt, "group": group}


def listed():
    return [
        # one token's hidden state: launches only
        {"name": "roundtrip_one_token", **_roundtrip(1, 4096, "bfloat16", "int8", 128)},
        # the hidden layer of a language model's feed-forward block, 8192 tokens
        {"name": "roundtrip_hidden_bf16", **_roundtrip(8192, 8192, "bfloat16", "int8", 64)},
        # a first convolution's output, 128 images of 55 x 55 pixels and 96 channels, single precision
        {"name": "roundtrip_conv1_fp32", **_roundtrip(128 * 55 * 55, 96, "float32", "e4m3", 32)},
        # an image classifier's last layer, 512 features to 1000 classes, batch 256: a small product in fp32
        {"name": "grad_classifier_fp32", **_linear(256, 512, 1000, "float32", "int8", 32, True)},
        # a square projection of a language model, 8192 tokens
        {"name": "grad_projection_bf16", **_linear(8192, 4096, 4096, "bfloat16", "int8", 128, False)},
        # a wide projection at a larger batch, 16384 tokens: the largest product
        {"name": "grad_expansion_bf16", **_linear(16384, 4096, 8192, "bfloat16", "e4m3", 64, False)},
        # a 1 x 1 convolution in a bottleneck, 64 images of 56 x 56: a long sum for a small result
        {"name": "grad_pointwise_bf16", **_linear(64 * 56 * 56, 256, 64, "bfloat16", "e4m3", 64, True)},
        # packed sequences of a half-precision run: nothing divides anything
        {"name": "grad_ragged_fp16", **_linear(4099, 2047, 1531, "float16", "int8", 64, True)},
        # the last stage of an image network on one image: latency
        {"name": "norm_one_image", **_norm(1, 49, 512, 32, "silu", "bfloat16")},
        # a block of an image generator, 128 x 128 latents, ten channels to a group
        {"name": "norm_latents_bf16", **_norm(8, 128 * 128, 320, 32, "silu", "bfloat16")},
        # small maps at a large batch: the last stage of a residual network in training, fp32
        {"name": "norm_train_7x7_fp32", **_train(256, 49, 512, 32, "relu", "float32", "int8", 32)},
        # the first stage of the same network, 112 x 112 pixels, mixed precision: the largest tensor
        {"name": "norm_train_112_bf16", **_train(256, 112 * 112, 64, 8, "silu", "bfloat16", "int8", 64)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dims(rng, hi):
    """A layer's width: mostly a multiple of 64, now and then anything."""
    v = _log(rng, 48, hi)
    return v if rng.random() < 0.4 else max(64, v // 64 * 64)


def draw(rng):
    op = rng.choice(["roundtrip", "linear_grad", "linear_grad", "norm", "norm_train"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    fmt, group = rng.choice(["int8", "e4m3"]), rng.choice([32, 64, 128])
    if op == "roundtrip":
        cols = _dims(rng, 12288)
        return _roundtrip(max(1, _log(rng, 4096, 60_000_000) // cols), cols, dtype, fmt, group)
    if op == "linear_grad":
        cols, outs = _dims(rng, 8192), _dims(rng, 8192)
        most = 16384 if dtype == "float32" else 200704
        rows = _log(rng, 1, max(64, min(most, 500_000_000_000 // (cols * outs))))
        return _linear(rows, cols, outs, dtype, fmt, group, rng.random() < 0.5)
    groups = rng.choice([1, 4, 8, 16, 32])
    channels = groups * _log(rng, 2, 1536 // groups)
    spatial = _log(rng, 1, 16384)
    batch = _log(rng, 1, max(1, min(256, 60_000_000 // (spatial * channels))))
    act = rng.choice(["none", "relu", "silu"])
    if op == "norm":
        return _norm(batch, spatial, channels, groups, act, dtype)
    return _train(batch, spatial, channels, groups, act, dtype, fmt, group)


# --- what a program has in hand ------------------------------------------------------------------------
def _activation(gen, rows, cols, dtype):
    """Hidden states: channels of different scales, a few of them much larger than the rest."""
    dev = torch.device("cuda", 0)
    scale = torch.exp(0.5 * torch.randn(cols, generator=gen, device=dev))
    scale[torch.rand(cols, generator=gen, device=dev) < 0.01] *= 20.0
    return (torch.randn(rows, cols, generator=gen, device=dev) * scale).to(_TYPES[dtype])


def prepare(case, seed):
    dev = torch.device("cuda", 0)
    gen = torch.Generator(device=dev).manual_seed(2011_09017 + seed)
    s = dict(case)
    if case["op"] == "roundtrip":
        s["x"] = _activation(gen, case["rows"], case["cols"], case["dtype"])
    elif case["op"] == "linear_grad":
        # the layer's input was stored in the forward pass: the program has its bytes
        codes, exps = _encode(_activation(gen, case["rows"], case["cols"], case["dtype"]), case["fmt"], case["group"])
        s["held"] = _pack(codes, exps)
        dy = torch.randn(case["rows"], case["outs"], generator=gen, device=dev)
        s["dy"] = (1e-2 * dy * torch.rand(case["rows"], 1, generator=gen, device=dev)).to(_TYPES[case["dtype"]])
    else:
        n, sp, c = case["batch"], case["spatial"], case["channels"]
        shift = torch.randn(c, generator=gen, device=dev)
        s["x"] = (_activation(gen, n * sp, c, "float32") + shift).view(n, sp, c).to(_TYPES[case["dtype"]])
        s["weight"] = 1.0 + 0.3 * torch.randn(c, generator=gen, device=dev)
        s["bias"] = 0.3 * torch.randn(c, generator=gen, device=dev)
        if case["op"] == "norm_train":
            s["dy"] = (1e-2 * torch.randn(n, sp, c, generator=gen, device=dev)).to(_TYPES[case["dtype"]])
    return s


# --- the plain forms -----------------------------------------------------------------------------------
def _groups(v, group, fill=0):
    """[rows, cols] -> [rows, groups of a row, group], short groups filled up."""
    rows, cols = v.shape
    short = -cols % group
    if short:
        v = torch.nn.functional.pad(v, (0, short), value=fill)
    return v.view(rows, -1, group)


def _power(e):
    """2^e in fp32, exactly, for -126 <= e <= 127 (a library's power function need not be)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _encode(x, fmt, group):
    """Codes (int8, or e4m3 numbers) [rows, cols] and exponents [rows, groups] of a matrix."""
    rows, cols = x.shape
    v = _groups(x.float(), group)
    amax = torch.where(torch.isfinite(v), v.abs(), 0.0).amax(2)
    frac, p = torch.frexp(amax)                                       # amax = frac * 2^p, 0.5 <= frac < 1
    if fmt == "int8":
        e = (p - 7 + (frac > 127.5 / 128).int()).clamp(-110, 121)
    else:
        e = (p - 9 + (frac > 448 / 512).int()).clamp(-110, 119)
    e = torch.where(amax == 0, -110, e)
    v = v * _power(-e)[:, :, None]
    finite = torch.isfinite(v)
    if fmt == "int8":
        codes = torch.where(finite, torch.round(v).clamp(-127, 127), -128.0).to(torch.int8)
    else:
        codes = torch.where(finite, v.clamp(-448, 448), float("nan")).to(torch.float8_e4m3fn)
    return codes.view(rows, -1)[:, :cols], e


def _decode(codes, exps, group):
    """The values that codes stand for, in fp32."""
    rows, cols = codes.shape
    v = codes.float()
    if codes.dtype == torch.int8:
        v = torch.where(v == -128, float("nan"), v)
    v = _groups(v, group) * _power(exps)[:, :, None]
    return v.view(rows, -1)[:, :cols]


def _pack(codes, exps):
    rows, cols = codes.shape
    n = rows * _pitch(cols)
    buf = torch.zeros((n + exps.numel() + 15) // 16 * 16, dtype=torch.uint8, device=codes.device)
    buf[:n].view(rows, -1)[:, :cols] = codes.contiguous().view(torch.uint8)
    buf[n:n + exps.numel()] = (exps + 127).to(torch.uint8).view(-1)
    return buf


def _unpack(buf, case):
    rows, cols = case["rows"], case["cols"]
    n, m = rows * _pitch(cols), -(-cols // case["group"])
    kind = torch.int8 if case["fmt"] == "int8" else torch.float8_e4m3fn
    codes = buf[:n].view(rows, -1)[:, :cols].contiguous().view(kind)
    return codes, buf[n:n + rows * m].view(rows, m).int() - 127


def _act(u, kind):
    return u * torch.sigmoid(u) if kind == "silu" else torch.where(u > 0, u, 0.0) if kind == "relu" else u


def _act_slope(u, kind):
    if kind == "silu":
        g = torch.sigmoid(u)
        return g * (1 + u * (1 - g))
    return torch.ones_like(u)


_EPS = 1e-5


def _per_channel(v, c):
    """[batch, groups] -> [batch, 1, channels]."""
    return v.repeat_interleave(c // v.shape[1], 1)[:, None, :]


def _moments(x, groups):
    """Mean and 1 / deviation of every (sample, group) of x[batch, spatial, channels]."""
    n, _, c = x.shape
    v = x.view(n, -1, groups, c // groups)
    mean = v.mean((1, 3))
    var = (v - mean[:, None, :, None]).square().mean((1, 3))
    return mean, 1 / torch.sqrt(var + _EPS)


def _normed(x, mean, rstd):
    return (x - _per_channel(mean, x.shape[2])) * _per_channel(rstd, x.shape[2])


def _norm_gradient(dy, x, mean, rstd, weight, bias, groups, act, positive):
    n, sp, c = x.shape
    per, r = c // groups, _per_channel(rstd, c)
    h = _normed(x, mean, rstd)
    du = torch.where(positive, dy, 0.0) if act == "relu" else dy * _act_slope(h * weight + bias, act)
    dh = du * weight
    a = dh.view(n, sp, groups, per).sum((1, 3)) / (sp * per)
    b = (dh * h).view(n, sp, groups, per).sum((1, 3)) / (sp * per)
    dx = r * (dh - _per_channel(a, c) - h * _per_channel(b, c))
    return dx, (du * h).sum((0, 1)), du.sum((0, 1))


def _plain(s):
    kind = _TYPES[s["dtype"]]
    if s["op"] == "roundtrip":
        return _decode(*_encode(s["x"], s["fmt"], s["group"]), s["group"]).to(kind)
    if s["op"] == "linear_grad":
        dy = s["dy"].float()
        dw = (dy.t() @ _decode(*_unpack(s["held"], s), s["group"])).to(kind)
        return (dw, dy.sum(0).to(kind)) if s["bias"] else dw
    x = s["x"].float()
    mean, rstd = _moments(x, s["groups"])
    c = s["channels"]
    y = _act(_normed(x, mean, rstd) * s["weight"] + s["bias"], s["act"]).to(kind)
    if s["op"] == "norm":
        return y
    held = _decode(*_encode(s["x"].view(-1, c), s["fmt"], s["group"]), s["group"]).view_as(x)
    positive = None
    if s["act"] == "relu":                                            # which side of the border: in 64 bits
        positive = _normed(held.double(), *_moments(x.double(), s["groups"])) * s["weight"] + s["bias"] > 0
    dx, dweight, dbias = _norm_gradient(s["dy"].float(), held, mean, rstd, s["weight"], s["bias"], s["groups"], s["act"],
                                        positive)
    return y, dx.to(kind), dweight, dbias


def run(state):
    if not own:
        return _plain(state)
    from paper_2011_09017_amd import operators as ops
    s = state
    if s["op"] == "roundtrip":
        return ops.byte_load(ops.byte_store(s["x"], s["fmt"], s["group"]))
    if s["op"] == "linear_grad":
        held = ops.ByteCheckpoint(s["held"], (s["rows"], s["cols"]), s["dy"].dtype, s["fmt"], s["group"])
        dw, db = ops.byte_linear_grad(s["dy"], held, bias=s["bias"])
        return (dw, db) if s["bias"] else dw
    if s["op"] == "norm":
        return ops.group_norm(s["x"], s["groups"], s["weight"], s["bias"], _EPS, s["act"])[0]
    y, stats, held = ops.group_norm(s["x"], s["groups"], s["weight"], s["bias"], _EPS, s["act"], save=s["fmt"],
                                    group=s["group"])
    dx, dweight, dbias = ops.group_norm_grad(s["dy"], held, stats, s["groups"], s["weight"], s["bias"], s["act"])
    return y, dx, dweight, dbias


def work(case):
    es = _bytes(case["dtype"])
    if case["op"] == "roundtrip":
        n = case["rows"] * case["cols"]                               # x in, held bytes out and in again, x' out
        return {"bytes": 2 * es * n + 2 * _held(case, case["rows"], case["cols"]), "flops": 4 * n}
    if case["op"] == "linear_grad":
        m, k, n = case["rows"], case["cols"], case["outs"]
        return {"bytes": es * m * n + _held(case, m, k) + es * n * k + (es * n if case["bias"] else 0),
                "flops": 2 * m * n * k + (m * n if case["bias"] else 0)}
    rows, c = case["batch"] * case["spatial"], case["channels"]
    if case["op"] == "norm":
        return {"bytes": 2 * es * rows * c + 8 * c, "flops": 12 * rows * c}
    return {"bytes": 4 * es * rows * c + 2 * _held(case, rows, c) + 24 * c, "flops": 40 * rows * c}


# --- from the definitions, in 64 bits ------------------------------------------------------------------
def _power64(e):
    return ((e + 1023) << 52).view(torch.float64)


def _held_values(x, fmt, group):
    """x' of x[rows, cols] in fp64, element by element from the definition."""
    rows, cols = x.shape
    v = x.double()
    which = torch.arange(cols, device=x.device) // group
    amax = torch.zeros(rows, int(which[-1]) + 1, dtype=torch.float64, device=x.device)
    amax = amax.scatter_reduce(1, which.expand(rows, -1), v.abs(), "amax")
    top = 127.5 if fmt == "int8" else 448.0
    # the smallest exponent for which the largest magnitude does not pass the largest code
    e = torch.ceil(torch.log2((amax / top).clamp_min(1e-300))).long()
    e = torch.where(amax > top * _power64(e), e + 1, e)
    e = torch.where(amax <= top * _power64(e - 1), e - 1, e).clamp(-110, 121 if fmt == "int8" else 119)
    unit = _power64(e)[:, which]
    v = v / unit
    if fmt == "int8":
        return torch.round(v).clamp(-127, 127) * unit
    step = _power64(torch.frexp(v)[1].clamp_min(-5).long() - 4)      # 3 bits behind the leading one; 2^-9 at the bottom
    return torch.round(v / step) * step * unit


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "roundtrip":
        return _held_values(s["x"], case["fmt"], case["group"])
    if case["op"] == "linear_grad":
        codes, exps = _unpack(s["held"], case)
        unit = _power64(exps.long()).repeat_interleave(case["group"], 1)[:, :case["cols"]]
        dy = s["dy"].double()
        dw = torch.mm(dy.t().contiguous(), codes.float().double() * unit)
        return (dw, dy.sum(0)) if case["bias"] else dw
    n, sp, c = s["x"].shape
    per = c // case["groups"]
    x = s["x"].double().view(n, sp, case["groups"], per)
    mean = x.mean((1, 3), keepdim=True)
    dev = ((x * x).mean((1, 3), keepdim=True) - mean * mean + _EPS).sqrt()
    w, b = (s[k].double().view(case["groups"], per) for k in ("weight", "bias"))
    u = (x - mean) / dev * w + b
    y = u / (1 + torch.exp(-u)) if case["act"] == "silu" else u.clamp_min(0) if case["act"] == "relu" else u
    y = y.reshape(n, sp, c)
    if case["op"] == "norm":
        return y
    h = (_held_values(s["x"].view(-1, c), case["fmt"], case["group"]).view_as(x) - mean) / dev
    u = h * w + b
    g = s["dy"].double().view_as(x)
    if case["act"] == "silu":
        t = torch.exp(-u)
        g = g * ((1 + t + u * t) / (1 + t) ** 2)
    elif case["act"] == "relu":
        g = torch.where(u > 0, g, 0.0)
    p, q = g.sum(1), (g * h).sum(1)                                   # per sample and channel
    a, b = ((v * w).sum(2)[:, None, :, None] / (sp * per) for v in (p, q))
    dx = ((g * w - a - h * b) / dev).reshape(n, sp, c)
    return y, dx, q.sum(0).view(c), p.sum(0).view(c)
