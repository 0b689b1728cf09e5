"""Group norm with an activation, channels last, forward and backward, against the formulas in float64.

Bounds, from the roundings that the kernels make (2^-24 each, relative to what is rounded; the sums of the
forward pass are in fp64):
  u = (x - mean) * (r * gamma) + beta      is off by at most 2^-21 * T, T = |gamma| r (|x| + |mean|) + |beta| (mean, the
                                           difference, r * gamma and the sum are rounded: four steps of these terms);
  y = act(u)                               by 1.1 of that (the steepest slope of u * sigmoid(u)) plus 2^-20 * (|u| + 1) * |y|
                                           for exp2 of a rounded argument and the reciprocal, and half a step of its type;
  du = dy * act'(u)                        by |dy| (0.5 * 2^-21 * T + 2^-20 (|u| + 1)) (the largest |act''| is 0.5);
  sums over k terms                        by k * 2^-24 * sum |terms| where a thread adds them in fp32, plus the terms' errors;
  dx                                       by r (that of du * |gamma|, those of A and of h * B) plus 2^-21 of their sizes.
"""
import math

import numpy as np
import pytest
import torch

import byte_reference as ref
from paper_2011_09017_amd import binding, operators as ops

TYPES = [torch.float32, torch.float16, torch.bfloat16]
EPS = 1e-5


def test_library_refusals():
    b, P = binding, 4096
    good = dict(batch=2, spatial=9, channels=24, groups=4, type=0, act=0, eps=1e-5)
    assert b.cmp_group_norm_work(b.cmp_norm_shape(**good)) > 0

    def both(s, x=P, y=P, gamma=None, stats=P, ck=None, cap=1 << 30, fmt=0, group=64, work=P, need=1 << 30):
        f = b.cmp_group_norm(0, s, x, gamma, None, y, stats, fmt, group, ck, cap, work, need, 0)
        g = b.cmp_group_norm_grad(0, s, P, None if ck else x, fmt, group, ck, cap, gamma, None, stats, y, P, P, work, need, 0)
        return f, g
    for bad in (dict(channels=0), dict(channels=8208), dict(groups=0), dict(groups=5), dict(channels=8192, groups=8192), dict(type=3),
                dict(act=3), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(batch=1 << 22),
                dict(spatial=1 << 31), dict(batch=1 << 16, spatial=1 << 16)):
        s = b.cmp_norm_shape(**{**good, **bad})
        assert b.cmp_group_norm_work(s) == 0, bad
        assert both(s) == (b.CMP_E_ARG, b.CMP_E_ARG), bad
    assert b.cmp_group_norm_work(b.cmp_norm_shape(**{**good, 'batch': 1})) == 0      # one pass, nothing between workgroups
    s = b.cmp_norm_shape(**good)
    need = b.cmp_group_norm_work(s)
    for kw in (dict(x=0), dict(x=P + 2), dict(y=0), dict(y=P + 1), dict(gamma=P + 2), dict(stats=P + 4), dict(work=P + 8), dict(work=0),
               dict(ck=P + 8), dict(ck=P, group=48), dict(ck=P, fmt=2)):
        assert both(s, **kw) == (b.CMP_E_ARG, b.CMP_E_ARG), kw
    assert both(s, need=need - 1) == (b.CMP_E_NOSPACE, b.CMP_E_NOSPACE)
    n = b.cmp_byte_bytes(b.cmp_byte_shape(18, 24, 0, 64))
    assert both(s, ck=P, cap=n - 1) == (b.CMP_E_NOSPACE, b.CMP_E_FORMAT)
    grad = lambda x, ck, stats=P: b.cmp_group_norm_grad(0, s, P, x, 0, 64, ck, n, None, None, stats, P, P, P, P, need, 0)  # noqa: E731
    assert grad(None, None) == grad(P, P) == grad(P, None, 0) == b.CMP_E_ARG


def test_sizes_past_32_bits_are_refused():
    """Fields of the C shape have 32 bits: what would wrap round to a legal size is refused."""
    with pytest.raises(ValueError, match="groups"):
        ops.group_norm(torch.empty(1, 8), (1 << 32) + 2)
    with pytest.raises(ValueError, match="channels"):
        ops.group_norm(torch.empty(0, (1 << 32) + 8), 2)
    with pytest.raises(ValueError, match="groups"):
        ops.group_norm(torch.empty(1, 8), -1)


def test_the_plan_keeps_to_what_a_launch_can_count():
    """2^21 samples of one position and 8192 channels: in segments of 1536 channels they would be 6 * 2^21 workgroups of 192, too
    many threads for one launch; the workspace is that of two passes, with a record of totals per sample and group."""
    shape = binding.cmp_norm_shape(1 << 21, 1, 8192, 128, binding.CMP_TYPE_BF, binding.CMP_ACT_NONE, 1e-5)
    assert binding.cmp_group_norm_work(shape) >= (1 << 21) * (16 * 128 + 8 * 8192)
    few = binding.cmp_norm_shape(1 << 10, 1, 8192, 128, binding.CMP_TYPE_BF, binding.CMP_ACT_NONE, 1e-5)
    assert (1 << 10) * 8 * 8192 <= binding.cmp_group_norm_work(few) < (1 << 10) * (16 * 128 + 8 * 8192)       # one pass


def test_formulas_against_differences():
    """The reference's gradients against differences of its forward pass (x' = x)."""
    gen = torch.Generator().manual_seed(0)
    x, dy = (torch.randn(2, 5, 12, generator=gen, dtype=torch.float64) for _ in range(2))
    w, b = (torch.randn(12, generator=gen, dtype=torch.float64) for _ in range(2))
    for act in ("none", "relu", "silu"):
        loss = lambda x, w, b: (ref.norm(x, 3, w, b, EPS, act)[0] * dy).sum()  # noqa: E731
        _, mean, rstd, _ = ref.norm(x, 3, w, b, EPS, act)
        grads = ref.norm_grad(dy, x, mean, rstd, w, b, act)[:3]
        for k, g in enumerate(grads):
            for i in range(0, g.numel(), 7):
                d = torch.zeros(g.numel(), dtype=torch.float64)
                d[i] = 1e-6
                up, down = ([v + s * d.view_as(v) if j == k else v for j, v in enumerate((x, w, b))] for s in (1, -1))
                assert float(loss(*up) - loss(*down)) / 2e-6 == pytest.approx(float(g.reshape(-1)[i]), rel=1e-5, abs=1e-7)


def _inputs(batch, spatial, channels, dtype, shift=1.0, seed=0):
    gen = torch.Generator().manual_seed(batch + spatial + channels + seed)
    x = torch.randn(batch, spatial, channels, generator=gen) * torch.exp(0.5 * torch.randn(channels, generator=gen))
    x = (x + shift * torch.randn(channels, generator=gen)).to(dtype).cuda()
    dy = torch.randn(batch, spatial, channels, generator=gen).to(dtype).cuda()
    w = (1 + 0.5 * torch.randn(channels, generator=gen)).cuda()
    b = (0.5 * torch.randn(channels, generator=gen)).cuda()
    return x, dy, w, b


def _within(got, want, tol, what):
    """Within the tolerance; past the type's largest finite value, the infinity that a cast gives."""
    most, got = torch.finfo(got.dtype).max, got.double().cpu()
    past = (want.abs() + tol > most) & (want * got > 0) & (got.abs() >= most)
    off = torch.where(past, 0.0, (got - want).abs())
    assert bool((off <= tol).all()), (what, float((off / tol).nan_to_num(posinf=1e30).max()))


def _rounding(got, want):
    return ref.HALF_STEP[got.dtype] * want.abs() * 1.001 + (2.0 ** -25 if got.dtype == torch.float16 else 1e-37)


def _spread(v, n, s, c):
    """[n, 1, groups, 1] -> [n, 1, c]."""
    return v.expand(n, 1, v.shape[2], c // v.shape[2]).reshape(n, 1, c)


def _check_forward(x, y, stats, groups, w, b, act):
    n, s, c = x.shape
    xd, wd, bd = x.double().cpu(), w.double().cpu(), b.double().cpu()
    want, mean, rstd, u = ref.norm(xd, groups, wd, bd, EPS, act)
    assert torch.allclose(stats[..., 0].cpu(), mean.view(n, groups), rtol=1e-12, atol=1e-12)
    assert torch.allclose(stats[..., 1].cpu(), rstd.view(n, groups), rtol=1e-8, atol=0)
    t = wd.abs() * _spread(rstd, n, s, c) * (xd.abs() + _spread(mean, n, s, c).abs()) + bd.abs()
    _within(y, want, 1.1 * 2.0 ** -21 * t + 2.0 ** -20 * (u.abs() + 1) * want.abs() + _rounding(y, want), "y")


def _check_backward(dy, xd, stats, groups, w, b, act, dx, dw, db):
    """Against the formulas with the kernels' own statistics; xd: the input that the backward pass sees."""
    n, s, c = dy.shape
    yd, wd, bd = dy.double().cpu(), w.double().cpu(), b.double().cpu()
    mean, rstd = (stats[..., k].cpu().view(n, 1, groups, 1) for k in (0, 1))
    want, want_w, want_b, du, h = ref.norm_grad(yd, xd, mean, rstd, wd, bd, act)
    r, u = _spread(rstd, n, s, c), h * wd + bd
    t = wd.abs() * r * (xd.abs() + _spread(mean, n, s, c).abs()) + bd.abs()
    eu, eh = 2.0 ** -21 * t, 2.0 ** -22 * r * (xd.abs() + _spread(mean, n, s, c).abs())
    ed = yd.abs() * (0.5 * eu + 2.0 ** -20 * (u.abs() + 1)) if act == "silu" else torch.zeros_like(yd)
    k = (s + 16) * 2.0 ** -24
    _within(db, want_b, (ed + k * du.abs()).sum((0, 1)) + 2.0 ** -24 * want_b.abs() + 1e-37, "dbias")
    _within(dw, want_w, (ed * h.abs() + du.abs() * eh + (k + 2.0 ** -22) * (du * h).abs()).sum((0, 1)) + 2.0 ** -24 * want_w.abs() + 1e-37,
            "dweight")

    def mean_of(v):
        return _spread(v.view(n, s, groups, -1).mean((1, 3), keepdim=True), n, s, c)
    g = wd.abs()
    ea = mean_of(g * (ed + (k + 2.0 ** -22) * du.abs()))
    eb = mean_of(g * (ed * h.abs() + du.abs() * eh + (k + 2.0 ** -21) * (du * h).abs()))
    size_a, size_b = mean_of(g * du.abs()), mean_of(g * (du * h).abs())
    tol = r * (g * ed + ea + h.abs() * eb + eh * size_b + 2.0 ** -21 * (g * du.abs() + size_a + h.abs() * size_b))
    _within(dx, want, tol + _rounding(dx, want), "dx")


SHAPES = [(1, 1, 1, 1), (1, 1, 8, 8), (2, 49, 512, 32), (3, 7, 30, 3), (1, 1000, 10, 1), (2, 3025, 96, 8), (5, 1, 64, 4), (1, 5, 8192, 4096),
          (2, 33, 8192, 1), (7, 13, 40, 4), (300, 4, 24, 2), (1, 4097, 320, 32), (2, 196, 1000, 125), (1, 2, 4100, 2),
          # two passes: groups narrower than a vector with the widest rows, rows of more than 512 vectors, and one group of all
          (1, 600, 8192, 4096), (2, 530, 4104, 171), (3, 1500, 30, 10), (1, 9000, 64, 1), (40, 600, 128, 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("batch,spatial,channels,groups", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act,save,group", [("none", None, 64), ("silu", "int8", 64), ("relu", "e4m3", 32), ("silu", None, 64), ("relu", "int8", 128),
                                            ("none", "e4m3", 128)])
def test_both_directions(batch, spatial, channels, groups, dtype, act, save, group):
    x, dy, w, b = _inputs(batch, spatial, channels, dtype)
    y, stats, ck = ops.group_norm(x, groups, w, b, EPS, act, save=save, group=group)
    assert y.dtype == dtype and y.shape == x.shape
    _check_forward(x, y, stats, groups, w, b, act)
    seen = x.double().cpu()
    if save is None:
        assert ck is None
    else:
        assert torch.equal(ck.buf, ops.byte_store(x, save, group).buf)       # the bytes of a store, to the last
        seen = torch.from_numpy(ref.held(ck)).view(x.shape)
    dx, dw, db = ops.group_norm_grad(dy, x if ck is None else ck, stats, groups, w, b, act)
    assert dx.dtype == dtype and dw.dtype == db.dtype == torch.float32
    _check_backward(dy, seen, stats, groups, w, b, act, dx, dw, db)
    # a second call gives the same bits
    again = ops.group_norm(x, groups, w, b, EPS, act, save=save, group=group)
    assert torch.equal(again[0], y) and torch.equal(again[1], stats)
    for p, q in zip(ops.group_norm_grad(dy, x if ck is None else ck, stats, groups, w, b, act), (dx, dw, db)):
        assert torch.equal(p, q)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,spatial,channels,groups", [(5000, 1, 40, 5), (2100, 2, 520, 130), (3000, 4, 96, 3), (2049, 7, 16, 16),
                                                           (2048, 16, 64, 2), (4097, 1, 4104, 1), (2500, 1, 7, 7)])
@pytest.mark.parametrize("dtype,act,save,group", [(torch.bfloat16, "silu", "int8", 32), (torch.float32, "relu", None, 64),
                                                  (torch.float16, "none", "e4m3", 128)])
def test_many_samples(batch, spatial, channels, groups, dtype, act, save, group):
    """The sums of the parameters are joined in two steps, groups of few values by a part of a wave."""
    test_both_directions(batch, spatial, channels, groups, dtype, act, save, group)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_without_parameters(act):
    x, dy, _, _ = _inputs(2, 50, 36, torch.bfloat16)
    one, zero = torch.ones(36, device="cuda"), torch.zeros(36, device="cuda")
    y, stats, _ = ops.group_norm(x, 6, act=act)
    assert torch.equal(y, ops.group_norm(x, 6, one, zero, act=act)[0])
    full = ops.group_norm_grad(dy, x, stats, 6, one, zero, act)
    for p, q in zip(ops.group_norm_grad(dy, x, stats, 6, act=act), full):
        assert torch.equal(p, q)
    dx, dw, db = ops.group_norm_grad(dy, x, stats, 6, act=act, params=False)
    assert torch.equal(dx, full[0]) and dw is None and db is None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("spatial", [20, 5000])
def test_mean_far_from_zero(dtype, spatial):
    """Deviations a thousandth of the mean: sums of squares in fp32 would lose the variance."""
    x, dy, w, b = _inputs(2, spatial, 24, torch.float32, shift=0.0)
    x = (x * 0.5 + 400.0).to(dtype)
    y, stats, _ = ops.group_norm(x, 4, w, b, EPS, "silu")
    _check_forward(x, y, stats, 4, w, b, "silu")
    dy = dy.to(dtype)
    _check_backward(dy, x.double().cpu(), stats, 4, w, b, "silu", *ops.group_norm_grad(dy, x, stats, 4, w, b, "silu"))


@pytest.mark.gpu
@pytest.mark.parametrize("spatial", [16, 3000])
def test_constant_groups_and_zeros(spatial):
    """No variance: h is 0, y is act(beta), dx is what the formula says with h = 0."""
    x = torch.full((2, spatial, 16), 3.0, device="cuda")
    x[1] = 0
    b = torch.linspace(-2, 2, 16, device="cuda")
    y, stats, ck = ops.group_norm(x, 4, None, b, EPS, "relu", save="int8", group=32)
    assert torch.equal(y, torch.relu(b).expand_as(y))
    dy = torch.randn(2, spatial, 16, generator=torch.Generator().manual_seed(2)).cuda()
    dx, dw, db = ops.group_norm_grad(dy, ck, stats, 4, None, b, "relu")
    _check_backward(dy, x.double().cpu(), stats, 4, torch.ones(16), b, "relu", dx, dw, db)


@pytest.mark.gpu
@pytest.mark.parametrize("spatial", [40, 5000])
def test_relu_border_is_decided_in_64_bits(spatial):
    """beta puts u next to zero for one of the codes' values in every channel: on which side each of those positions lies
    is counted by dbias exactly."""
    x, _, w, _ = _inputs(1, spatial, 32, torch.float32)
    x = torch.round(x * 8) / 8                                   # many equal values
    _, stats, ck = ops.group_norm(x, 4, w, None, EPS, "none", save="int8", group=32)
    mean, rstd = (stats[..., k].cpu().view(1, 1, 4, 1) for k in (0, 1))
    held = torch.from_numpy(ref.held(ck)).view(x.shape)
    h = ref.normed(held, mean, rstd)
    wd = w.double().cpu()
    b = -(h[:, 0] * wd).float()[0].cuda()                        # u of position 0: a rounding of beta from zero
    u = h * wd + b.double().cpu()
    dy = torch.ones_like(x)
    _, _, db = ops.group_norm_grad(dy, ck, stats, 4, w, b, "relu")
    assert torch.equal(db.double().cpu(), (u > 0).double().sum((0, 1)))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("spatial", [30, 3000])
def test_nan_spoils_its_group_only(act, spatial):
    x, dy, w, b = _inputs(2, spatial, 32, torch.float32)
    x[1, 3, 9] = float("nan")
    x[0, 5, 31] = float("inf")
    y, stats, ck = ops.group_norm(x, 4, w, b, EPS, act, save="int8", group=32)
    bad = torch.zeros(2, 1, 32, dtype=torch.bool)
    bad[1, :, 8:16] = bad[0, :, 24:] = True
    assert torch.equal(torch.isnan(y).cpu(), bad.expand_as(y))
    dx, dw, db = ops.group_norm_grad(dy, ck, stats, 4, w, b, act)
    assert torch.equal(~torch.isfinite(dx).cpu(), bad.expand_as(dx))
    per_channel = bad.any(0)[0]
    assert torch.equal(torch.isnan(dw).cpu(), per_channel)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(0, 4, 8), (3, 0, 8)])
def test_empty(shape):
    x = torch.zeros(shape, device="cuda")
    y, stats, ck = ops.group_norm(x, 2, save="int8")
    dx, dw, db = ops.group_norm_grad(x, ck, stats, 2)
    assert y.shape == dx.shape == x.shape and not dw.any() and not db.any()


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """More than 2^32 elements: the last sample against the formulas, its checkpoint against a store."""
    n, s, c, groups = 3, 200_000, 8192, 4
    assert n * s * c > 2 ** 32
    x = torch.zeros(n, s, c, dtype=torch.bfloat16, device="cuda")
    for k in range(0, s, 20_000):
        x[-1, k:k + 20_000] = torch.randn(20_000, c, device="cuda", generator=torch.Generator("cuda").manual_seed(k)) + 2
    y, stats, ck = ops.group_norm(x, groups, save="int8", group=128)
    last = x[-1].view(s, groups, c // groups)
    mean = torch.stack([last[:, g].sum(dtype=torch.float64) for g in range(groups)]) / (s * (c // groups))
    assert torch.allclose(stats[-1, :, 0], mean, rtol=1e-10, atol=0)
    tail = x[-1, -50:].double().cpu().view(1, 50, c)
    want = ref.normed(tail, *(stats[-1:, :, k].cpu().view(1, 1, groups, 1) for k in (0, 1)))
    got = y[-1, -50:].double().cpu().view(1, 50, c)
    assert bool(((got - want).abs() <= 2.0 ** -8 * 1.001 * want.abs() + 2.0 ** -19).all())
    codes = ck.buf[n * s * c - 50 * c:n * s * c].cpu().numpy().reshape(50, c)
    want_codes, _ = ref.encode(tail[0].numpy(), "int8", 128)
    assert np.array_equal(codes, want_codes)
    del y
    dx, dw, db = ops.group_norm_grad(x, ck, stats, groups)
    h = want[0]                                                  # dy = x here
    held = torch.from_numpy(ref.decode(*ref.encode(tail[0].numpy(), "int8", 128), "int8", 128)).view(1, 50, c)
    h = ref.normed(held, *(stats[-1:, :, k].cpu().view(1, 1, groups, 1) for k in (0, 1)))
    a = mean.cpu().view(1, 1, groups, 1)
    b = torch.stack([(last[:, g].float() * (last[:, g].float() - float(mean[g])) * float(stats[-1, g, 1])).sum(dtype=torch.float64)
                     for g in range(groups)]).cpu().view(1, 1, groups, 1) / (s * (c // groups))
    dx_want = (stats[-1:, :, 1].cpu().view(1, 1, groups, 1) * (tail.view(1, 50, groups, -1) - a - h.view(1, 50, groups, -1) * b)).reshape(1, 50, c)
    # B was taken from x instead of x': they differ by half a code's step per value, far less in the mean
    assert bool(((dx[-1, -50:].double().cpu().view(1, 50, c) - dx_want).abs() <= 2.0 ** -8 * dx_want.abs() + 0.01).all())


@pytest.mark.gpu
def test_refusals_on_the_gpu():
    x, dy, w, b = _inputs(2, 9, 24, torch.bfloat16)
    y, stats, ck = ops.group_norm(x, 4, w, b, save="int8")
    for call in (lambda: ops.group_norm(x.transpose(1, 2), 4), lambda: ops.group_norm(x[:, :, 0], 4)[0] if False else ops.group_norm(x[0, 0], 4),
                 lambda: ops.group_norm(x, 4, w.bfloat16()), lambda: ops.group_norm(x, 4, w[:23]), lambda: ops.group_norm(x, 4, w.cpu()),
                 lambda: ops.group_norm(x, 4, act="gelu"), lambda: ops.group_norm(x, 4, save="int4"), lambda: ops.group_norm(x, 4, save="int8", group=16),
                 lambda: ops.group_norm_grad(dy[:1], ck, stats, 4), lambda: ops.group_norm_grad(dy.float(), x, stats, 4),
                 lambda: ops.group_norm_grad(dy, ck, stats.float(), 4), lambda: ops.group_norm_grad(dy, ck, stats, 8),
                 lambda: ops.group_norm_grad(dy, ck, stats[:1], 4), lambda: ops.group_norm(x.cpu(), 4)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ops.group_norm(x, 5), lambda: ops.group_norm(x, 0), lambda: ops.group_norm(x, 4, eps=0.0),
                 lambda: ops.group_norm_grad(dy, ck._replace(buf=ck.buf[:16]), stats, 4)):
        with pytest.raises(binding.CmpError):
            call()
