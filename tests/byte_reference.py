"""Byte checkpoints and the operators on them in 64 bits on the CPU, from the definitions in include/cmpz.h."""
import numpy as np
import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # of a rounding, relative


def e4m3_values():
    """Values of the codes 0 .. 0x7e (non-negative, ascending)."""
    v = []
    for c in range(0x7f):
        e, m = c >> 3, c & 7
        v.append((8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9)
    return np.array(v)


def _nearest_even(v, table):
    """Index into an ascending table whose neighbours' midpoints go to the even index."""
    mid = (table[1:] + table[:-1]) / 2
    i = np.searchsorted(mid, v, side="left")                 # v on a midpoint: the lower index
    at = np.minimum(i, len(mid) - 1)
    return np.where((i < len(mid)) & (v == mid[at]) & (i % 2 == 1), i + 1, i)


def encode(x, fmt, group):
    """(codes uint8 [rows, cols], exponents int [rows, groups]) of a float64 matrix."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    ng = -(-cols // group)
    codes, exps = np.zeros((rows, cols), np.uint8), np.full((rows, ng), -110)
    top, cap = (127.5, 121) if fmt == "int8" else (448.0, 119)
    table = e4m3_values()
    for g in range(ng):
        v = x[:, g * group:(g + 1) * group]
        fine = np.isfinite(v)
        amax = np.where(fine, np.abs(v), 0.0).max(1)
        e = np.frexp(amax / top)[1]                            # amax / top = f * 2^e, 0.5 <= f < 1 ...
        e = np.where(amax == top * 2.0 ** (e - 1.0), e - 1, e)   # ... unless it is a power of two itself
        e = np.clip(np.where(amax == 0, -110, e), -110, cap)
        t = np.where(fine, v, 0.0) * 2.0 ** -e[:, None].astype(np.float64)
        if fmt == "int8":
            c = np.clip(np.rint(t), -127, 127).astype(np.int8).view(np.uint8)
            c = np.where(fine, c, 0x80)
        else:
            c = _nearest_even(np.minimum(np.abs(t), 448.0), table).astype(np.uint8)
            c = np.where(np.signbit(t), c | 0x80, c)
            c = np.where(fine, c, 0x7f)
        codes[:, g * group:(g + 1) * group] = c
        exps[:, g] = e
    return codes, exps


def decode(codes, exps, fmt, group):
    cols = codes.shape[1]
    if fmt == "int8":
        v = codes.view(np.int8).astype(np.float64)
        v[codes == 0x80] = np.nan
    else:
        v = np.append(e4m3_values(), np.nan)[codes & 0x7f]
        v = np.where(codes & 0x80, -v, v)
    return v * np.repeat(2.0 ** exps.astype(np.float64), group, axis=1)[:, :cols]


def split(buf, rows, cols, group):
    """(codes, padding, exponents, tail) of a checkpoint's bytes."""
    pitch, ng = (cols + 15) // 16 * 16, -(-cols // group)
    b = np.asarray(buf)
    c = b[:rows * pitch].reshape(rows, pitch)
    e = b[rows * pitch:rows * (pitch + ng)].reshape(rows, ng)
    total = (rows * (pitch + ng) + 15) // 16 * 16
    return c[:, :cols], c[:, cols:], e.astype(np.int64) - 127, b[rows * (pitch + ng):total]


def held(ck):
    """x' of a ByteCheckpoint, float64 [rows, cols]."""
    codes, _, exps, _ = split(ck.buf.cpu().numpy(), ck.rows, ck.cols, ck.group)
    return decode(np.ascontiguousarray(codes), exps, ck.fmt, ck.group)


def sigmoid(u):
    return 1 / (1 + torch.exp(-u))


def norm(x, groups, weight, bias, eps, act):
    """y, mean and 1 / deviation [batch, 1, groups, 1], u of a float64 tensor [batch, spatial, channels]."""
    n, s, c = x.shape
    v = x.view(n, s, groups, c // groups)
    mean = v.mean((1, 3), keepdim=True)
    rstd = 1 / (((v - mean) ** 2).mean((1, 3), keepdim=True) + eps).sqrt()
    u = normed(x, mean, rstd) * weight + bias
    y = u * sigmoid(u) if act == "silu" else torch.relu(u) if act == "relu" else u
    return y, mean, rstd, u


def normed(x, mean, rstd):
    n, s, c = x.shape
    return ((x.view(n, s, mean.shape[2], -1) - mean) * rstd).reshape(n, s, c)


def norm_grad(dy, x, mean, rstd, weight, bias, act):
    """dx, dweight, dbias, du and h from the formulas, float64."""
    n, s, c = x.shape
    groups = mean.shape[2]
    h = normed(x, mean, rstd)
    u = h * weight + bias
    if act == "silu":
        g = sigmoid(u)
        du = dy * g * (1 + u * (1 - g))
    else:
        du = torch.where(u > 0, dy, torch.zeros_like(dy)) if act == "relu" else dy
    d = (du * weight).view(n, s, groups, -1)
    a, b = d.mean((1, 3), keepdim=True), (d * h.view_as(d)).mean((1, 3), keepdim=True)
    dx = (rstd * (d - a - h.view_as(d) * b)).reshape(n, s, c)
    return dx, (du * h).sum((0, 1)), du.sum((0, 1)), du, h
