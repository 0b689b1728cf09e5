"""Group norm of values far from zero, fp32: the error may grow with h = (x - mean) / deviation, not with mean / deviation.

Bounds.  x - mean is formed from the mean's fp32 value hi and what is left of it, lo, |lo| <= 2^-24 |mean|; with r = 1 / deviation
  h      takes three roundings of (x - hi) r and one each of lo r and of the sum: 4 * 2^-24 q, q = |h| + 2^-23 |mean| r;
  u      takes the product with gamma and the sum with beta (or r * gamma, lo r gamma and theirs): 2^-21 (|gamma| q + |beta|);
  r      comes from fp64 sums of squares as long as the variance and eps are 2^-16 of them: a value passes through some 200
         additions here, 200 * 2^-53 * 2^16 / 2 < 1e-9.  Otherwise from squares of differences from a value v near the mean, at
         worst one value of the group, sqrt(k) deviations from its mean for k values: 200 k 2^-53 / 2 < 1e-9;
  mean   is a sum of values or such a value and a sum of differences from it: at most k 2^-53 D, D the largest difference from the
         group's first value, and 1e-13 of itself for the sums of values as they are and for the reference's.
Everything behind h and u is as in the tests near zero."""
import pytest
import torch

import byte_reference as ref
from paper_2011_09017_amd import operators as ops

EPS = 1e-5


def _wide(v, n, c):
    return v.expand(n, 1, v.shape[2], c // v.shape[2]).reshape(n, 1, c)


def _near(got, want, tol, what):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), (what, float((off / tol.clamp_min(1e-300)).max()))


def _rounding(got, want):
    return ref.HALF_STEP[got.dtype] * want.abs() * 1.001 + 1e-37


def _check(x, dy, groups, w, b, act, save=None):
    n, s, c = x.shape
    xd, yd, wd, bd = (t.double().cpu() for t in (x, dy, w, b))
    y, stats, ck = ops.group_norm(x, groups, w, b, EPS, act, save=save)
    want, mean, rstd, u = ref.norm(xd, groups, wd, bd, EPS, act)
    v = xd.view(n, s, groups, -1)
    far = s * v.shape[3] * 2.0 ** -53 * (v - v[:, :1, :, :1]).abs().amax((1, 3))
    assert bool(((stats[..., 0].cpu() - mean.view(n, groups)).abs() <= far + 1e-13 * mean.view(n, groups).abs()).all())
    assert torch.allclose(stats[..., 1].cpu(), rstd.view(n, groups), rtol=1e-8, atol=0)
    r, low = _wide(rstd, n, c), 2.0 ** -23 * _wide(mean.abs() * rstd, n, c)
    eu = 2.0 ** -21 * (wd.abs() * (ref.normed(xd, mean, rstd).abs() + low) + bd.abs())
    _near(y, want, 1.1 * eu + 2.0 ** -20 * (u.abs() + 1) * want.abs() + _rounding(y, want), "y")

    seen = xd if ck is None else torch.from_numpy(ref.held(ck)).view(x.shape)
    dx, dw, db = ops.group_norm_grad(dy, x if ck is None else ck, stats, groups, w, b, act)
    mean, rstd = (stats[..., k].cpu().view(n, 1, groups, 1) for k in (0, 1))
    want, want_w, want_b, du, h = ref.norm_grad(yd, seen, mean, rstd, wd, bd, act)
    u, g = h * wd + bd, wd.abs()
    eh, eu = 2.0 ** -22 * (h.abs() + low), 2.0 ** -21 * (g * (h.abs() + low) + bd.abs())
    ed = yd.abs() * (0.5 * eu + 2.0 ** -20 * (u.abs() + 1)) if act == "silu" else torch.zeros_like(yd)
    k = (s + 16) * 2.0 ** -24

    def mean_of(v):
        return _wide(v.view(n, s, groups, -1).mean((1, 3), keepdim=True), n, c)
    ea = mean_of(g * (ed + (k + 2.0 ** -22) * du.abs()))
    eb = mean_of(g * (ed * h.abs() + du.abs() * eh + (k + 2.0 ** -21) * (du * h).abs()))
    size_a, size_b = mean_of(g * du.abs()), mean_of(g * (du * h).abs())
    _near(db, want_b, (ed + k * du.abs()).sum((0, 1)) + 2.0 ** -24 * want_b.abs() + 1e-37, "dbias")
    _near(dw, want_w, (ed * h.abs() + du.abs() * eh + (k + 2.0 ** -22) * (du * h).abs()).sum((0, 1)) + 2.0 ** -24 * want_w.abs() + 1e-37, "dweight")
    tol = r * (g * ed + ea + h.abs() * eb + eh * size_b + 2.0 ** -21 * (g * du.abs() + size_a + h.abs() * size_b))
    _near(dx, want, tol + _rounding(dx, want), "dx")


# one pass and two, groups of one to many channels, a multiple of eight or not, several samples
SHAPES = [(2, 49, 512, 32), (3, 7, 30, 3), (300, 4, 24, 2), (5, 1, 64, 4), (2, 33, 1024, 1), (4, 20, 36, 18), (70, 1, 40, 1),
          (3, 1500, 30, 10), (1, 4097, 320, 32), (2, 3025, 96, 8), (2, 530, 4104, 171), (1, 9000, 64, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("mean,dev", [(1e5, 0.05), (-3e6, 2.0), (1e-3, 1e-7), (64.0, 1.0)])
@pytest.mark.parametrize("batch,spatial,channels,groups", SHAPES)
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_far_from_zero(batch, spatial, channels, groups, mean, dev, act):
    gen = torch.Generator().manual_seed(batch + spatial + channels)
    x = (mean + dev * torch.randn(batch, spatial, channels, generator=gen, dtype=torch.float64)).float().cuda()
    dy = torch.randn(batch, spatial, channels, generator=gen).cuda()
    w, b = (1 + 0.5 * torch.randn(channels, generator=gen)).cuda(), (0.5 * torch.randn(channels, generator=gen)).cuda()
    _check(x, dy, groups, w, b, act)


@pytest.mark.gpu
@pytest.mark.parametrize("save", ["int8", "e4m3"])
@pytest.mark.parametrize("batch,spatial,channels,groups", [(2, 49, 512, 32), (3, 7, 30, 3), (1, 4097, 320, 32)])
def test_far_from_zero_from_codes(batch, spatial, channels, groups, save):
    """The codes of such values are coarse, but what they stand for enters exactly."""
    gen = torch.Generator().manual_seed(1)
    x = (500 + torch.randn(batch, spatial, channels, generator=gen, dtype=torch.float64)).float().cuda()
    dy = torch.randn(batch, spatial, channels, generator=gen).cuda()
    w, b = (1 + 0.5 * torch.randn(channels, generator=gen)).cuda(), (0.5 * torch.randn(channels, generator=gen)).cuda()
    _check(x, dy, groups, w, b, "silu", save)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [0.1, 1e6 + 0.3, -3e20, 3e38])
@pytest.mark.parametrize("batch,spatial,channels,groups", SHAPES)
def test_equal_values(batch, spatial, channels, groups, value):
    """No variance whatever the value: the mean is the value, r is 1 / sqrt(eps) to the bound above, y is beta, h is 0."""
    x = torch.full((batch, spatial, channels), value, device="cuda")
    b = torch.linspace(-2, 2, channels, device="cuda")
    y, stats, _ = ops.group_norm(x, groups, None, b, EPS)
    assert torch.equal(y, b.expand_as(y)) and bool((stats[..., 0] == float(x[0, 0, 0])).all())
    assert torch.allclose(stats[..., 1].cpu(), torch.full((batch, groups), EPS ** -0.5, dtype=torch.float64), rtol=1e-8, atol=0)
    assert not ops.group_norm(x, groups)[0].any()                 # without beta: zeros
    dy = torch.randn(x.shape, generator=torch.Generator().manual_seed(2)).cuda()
    dx, dw, db = ops.group_norm_grad(dy, x, stats, groups, None, b)
    assert not dw.any()
    a = dy.double().cpu().view(batch, spatial, groups, -1)
    r, mean = EPS ** -0.5, a.mean((1, 3), keepdim=True)
    tol = r * ((spatial + 32) * 2.0 ** -24 * a.abs().mean((1, 3), keepdim=True) + 2.0 ** -22 * (a - mean).abs() + 2.0 ** -23 * a.abs())
    assert bool(((dx.double().cpu().view(a.shape) - r * (a - mean)).abs() <= tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("batch,spatial,channels,groups", SHAPES)
def test_first_value_far_from_the_others(batch, spatial, channels, groups):
    """The value that the sums are taken about is 10^4 deviations from the rest: the bounds hold as they are."""
    gen = torch.Generator().manual_seed(3)
    x = 2 + torch.randn(batch, spatial, channels, generator=gen)
    x.view(batch, spatial, groups, -1)[:, 0, :, 0] = 1e4
    dy = torch.randn(batch, spatial, channels, generator=gen).cuda()
    w, b = (1 + 0.5 * torch.randn(channels, generator=gen)).cuda(), (0.5 * torch.randn(channels, generator=gen)).cuda()
    _check(x.cuda(), dy, groups, w, b, "silu")


@pytest.mark.gpu
@pytest.mark.parametrize("spatial", [40, 3000])
@pytest.mark.parametrize("channels,groups", [(64, 8), (60, 4), (40, 20)])
def test_groups_far_from_zero_beside_others(spatial, channels, groups):
    """One group of a workgroup far from zero, one spoilt by a NaN, one by an infinity: the others and the far one are right, and
    the NaNs stay in their groups."""
    gen = torch.Generator().manual_seed(4)
    per = channels // groups
    x = torch.randn(2, spatial, channels, generator=gen)
    x[0, :, per:2 * per] += 1e5
    x[1, 3, 2 * per] = float("nan")
    x[1, spatial - 1, 4 * per - 1] = float("inf")
    x = x.cuda()
    y, stats, _ = ops.group_norm(x, groups)
    bad = torch.zeros(2, 1, channels, dtype=torch.bool)
    bad[1, :, 2 * per:4 * per] = True
    assert torch.equal(torch.isnan(y).cpu(), bad.expand_as(y))
    xd = torch.where(bad, torch.zeros(1, dtype=torch.float64), x.double().cpu())
    want, mean, rstd, _ = ref.norm(xd, groups, torch.ones(channels, dtype=torch.float64), torch.zeros(channels, dtype=torch.float64), EPS, "none")
    low = 2.0 ** -23 * _wide(mean.abs() * rstd, 2, channels)
    good = torch.where(bad, want, y.double().cpu())
    assert bool(((good - want).abs() <= 2.0 ** -21 * (want.abs() + low) + 2.0 ** -24 * want.abs() + 1e-37).all())


@pytest.mark.gpu
@pytest.mark.parametrize("spatial", [49, 3000])
def test_replays_near_and_far_from_zero(spatial):
    """Captured once on values near zero, replayed on values far from it and back: the eager results every time."""
    gen = torch.Generator().manual_seed(5)
    sets = [[(far + torch.randn(3, spatial, 96, generator=gen)).cuda(), torch.randn(3, spatial, 96, generator=gen).cuda()] for far in (0.0, 1e4, 3e6)]
    w, b = torch.rand(96, generator=gen).cuda() + 0.5, torch.randn(96, generator=gen).cuda()

    def step(x, dy):
        y, stats, _ = ops.group_norm(x, 8, w, b, EPS, "silu")
        return [y, stats, *ops.group_norm_grad(dy, x, stats, 8, w, b, "silu")]
    want = [[t.clone() for t in step(*s)] for s in sets]
    ins = [t.clone() for t in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*ins)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        outs = step(*ins)
    for v in (1, 0, 2, 1, 0):
        for a, s in zip(ins, sets[v]):
            a.copy_(s)
        g.replay()
        torch.cuda.synchronize()
        for t, u in zip(outs, want[v]):
            assert torch.equal(t, u)
        step(*sets[(v + 1) % 3])
        torch.cuda.synchronize()
