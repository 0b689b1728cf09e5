"""Weight and bias gradient of a linear layer from its input's byte checkpoint, against float64.

Bound: every product is exact, so a result is off by its sum's roundings and its last one.  A sum of t terms in fp32
(t = rows, twice that for fp16 and three times for fp32, plus the partial sums that are joined) is off by at most
(t + 64) * 2^-23 * sum |terms|, with a whole step per addition allowed for the matrix units' alignment of
their terms; the last rounding by half a step of the output type.
"""
import numpy as np
import pytest
import torch

import byte_reference as ref
from paper_2011_09017_amd import binding, operators as ops

TERMS = {torch.bfloat16: 1, torch.float16: 2, torch.float32: 3}


def test_library_refusals():
    b, P = binding, 4096
    s = b.cmp_byte_shape(64, 40, 0, 32)
    n = b.cmp_byte_bytes(s)
    good = dict(ck=P, bytes=n, dy=P, type=2, outs=24, ld=24, dw=P, db=None, out=2, work=P, need=1 << 30)

    def call(**kw):
        a = {**good, **kw}
        return b.cmp_byte_linear_grad(0, s, a["ck"], a["bytes"], a["dy"], a["type"], a["outs"], a["ld"], a["dw"], a["db"], a["out"],
                                      False, a["work"], a["need"], 0)
    for kw in (dict(ck=0), dict(ck=P + 4), dict(dy=0), dict(dy=P + 1), dict(type=3), dict(outs=1 << 31), dict(ld=23), dict(dw=0),
               dict(dw=P + 1), dict(db=P + 1), dict(out=1), dict(out=3), dict(ld=(1 << 24) + 1)):
        assert call(**kw) == b.CMP_E_ARG, kw
    assert call(bytes=n - 1) == b.CMP_E_FORMAT
    for rows, cols, outs in ((0, 0, 0), (5, 0, 3), (5, 3, 0), (0, 3, 3), (1, 1, 1)):
        assert b.cmp_byte_linear_grad_work(b.cmp_byte_shape(rows, cols, 0, 32), outs, 0) == 0
    big = b.cmp_byte_shape(1 << 20, 40, 0, 32)
    need = b.cmp_byte_linear_grad_work(big, 24, 2)
    assert need > 0 and need % 4 == 0
    args = (P, 1 << 40, P, 2, 24, 24, P, None, 2, False)
    assert b.cmp_byte_linear_grad(0, big, *args, P, need - 1, 0) == b.CMP_E_NOSPACE
    assert b.cmp_byte_linear_grad(0, big, *args, 0, need, 0) == b.CMP_E_ARG
    assert b.cmp_byte_linear_grad(0, big, *args, P + 8, need, 0) == b.CMP_E_ARG


def _case(rows, cols, outs, dtype, fmt, group, seed=0):
    gen = torch.Generator().manual_seed(rows + 3 * cols + 7 * outs + seed)
    x = (torch.randn(rows, cols, generator=gen) * torch.exp(torch.randn(cols, generator=gen))).to(dtype).cuda()
    dy = (torch.randn(rows, outs, generator=gen) * torch.exp(torch.randn(rows, 1, generator=gen))).to(dtype).cuda()
    return ops.byte_store(x, fmt, group), dy


def _want(dy, ck):
    y, x = dy.double().cpu().reshape(-1, dy.shape[-1]), torch.from_numpy(ref.held(ck))
    return y.t() @ x, y.abs().t() @ x.abs(), y.sum(0), y.abs().sum(0)


def _close(got, want, size, terms):
    tol = (terms + 64) * 2.0 ** -23 * size + ref.HALF_STEP[got.dtype] * want.abs() * 1.001 + 1e-37
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25                                  # half a step among its smallest numbers
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


SHAPES = [(1, 1, 1), (1, 5, 7), (2, 128, 128), (33, 17, 130), (64, 96, 40), (257, 255, 129), (31, 512, 1000), (4099, 40, 64), (700, 300, 520),
          (20000, 64, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,outs", SHAPES)
@pytest.mark.parametrize("dtype", list(TERMS))
@pytest.mark.parametrize("fmt,group", [("int8", 32), ("e4m3", 64), ("int8", 128)])
def test_gradients(rows, cols, outs, dtype, fmt, group):
    ck, dy = _case(rows, cols, outs, dtype, fmt, group)
    want, size, want_b, size_b = _want(dy, ck)
    terms = rows * TERMS[dtype]
    dw, db = ops.byte_linear_grad(dy, ck, bias=True)
    assert dw.dtype == dtype and db.dtype == dtype
    _close(dw, want, size, terms)
    _close(db, want_b, size_b, terms)
    again, none = ops.byte_linear_grad(dy, ck)
    assert none is None and torch.equal(again, dw)             # the same bits, with the bias or without
    wide, wide_b = ops.byte_linear_grad(dy, ck, bias=True, dtype=torch.float32)
    _close(wide, want, size, terms)
    _close(wide_b, want_b, size_b, terms)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,outs", [(4099, 2047, 1531), (1000, 520, 776), (2500, 64, 2056), (3000, 1100, 70), (1537, 1025, 263),
                                            (300, 4000, 3), (2000, 9, 520), (70000, 8, 2), (3001, 257, 7), (5000, 1, 1), (2000, 100, 4)])
@pytest.mark.parametrize("dtype", list(TERMS))
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_larger_products(rows, cols, outs, dtype, fmt):
    """Every size of tile, several ranges of rows, edges that nothing divides, a NaN in one column; float64 on the GPU."""
    ck, dy = _case(rows, cols, outs, dtype, fmt, 64)
    nan_at = (rows - 1) * ((cols + 15) // 16 * 16) + cols // 2
    ck.buf[nan_at] = 0x80 if fmt == "int8" else 0x7f
    x = ops.byte_load(ck, dtype=torch.float32).double()
    assert int(torch.isnan(x).sum()) == 1
    fine = torch.arange(cols, device="cuda") != cols // 2
    x = torch.nan_to_num(x)
    y = dy.double()
    want, size = torch.mm(y.t().contiguous(), x), torch.mm(y.abs().t().contiguous(), x.abs())
    start = torch.randn(outs, cols, generator=torch.Generator().manual_seed(1)).cuda()
    dw, db = ops.byte_linear_grad(dy, ck, bias=True)
    assert bool(torch.isnan(dw[:, ~fine]).all()) and bool(torch.isfinite(dw[:, fine]).all())
    _close(dw[:, fine], want[:, fine].cpu(), size[:, fine].cpu(), rows * TERMS[dtype])
    _close(db, y.sum(0).cpu(), y.abs().sum(0).cpu(), rows * TERMS[dtype])
    sums, _ = ops.byte_linear_grad(dy, ck, out=start.clone(), accumulate=True)
    _close(sums[:, fine], (want + start.double())[:, fine].cpu(), (size + start.abs().double())[:, fine].cpu(), rows * TERMS[dtype] + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TERMS))
@pytest.mark.parametrize("rows,cols,outs", [(40, 70, 33), (9000, 64, 48)])
def test_accumulates(dtype, rows, cols, outs):
    ck, dy = _case(rows, cols, outs, dtype, "int8", 64)
    want, size, want_b, size_b = _want(dy, ck)
    start = torch.randn(outs, cols, generator=torch.Generator().manual_seed(1)).cuda()
    start_b = torch.randn(outs, generator=torch.Generator().manual_seed(2)).cuda()
    for kind in {torch.float32, dtype}:
        dw, db = start.to(kind), start_b.to(kind)
        w0, b0 = dw.double().cpu(), db.double().cpu()
        out, out_b = ops.byte_linear_grad(dy, ck, out=dw, out_bias=db, accumulate=True)
        assert out is dw and out_b is db
        _close(dw, want + w0, size + w0.abs(), rows * TERMS[dtype] + 1)
        _close(db, want_b + b0, size_b + b0.abs(), rows * TERMS[dtype] + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TERMS))
def test_strided_unaligned_and_contained(dtype):
    """dY inside a larger matrix of infinities at an odd offset; nothing outside dW and db is written."""
    ck, dy = _case(77, 50, 45, dtype, "int8", 32)
    big = torch.full((77, 61), float("inf"), dtype=dtype, device="cuda")
    big[:, 3:48] = dy
    guard = torch.full((45 * 50 + 64,), 7.0, dtype=dtype, device="cuda")
    guard_b = torch.full((45 + 64,), 7.0, dtype=dtype, device="cuda")
    ref_w, ref_b = ops.byte_linear_grad(dy, ck, bias=True)
    ops.byte_linear_grad(big[:, 3:48], ck, out=guard[1:2251].view(45, 50), out_bias=guard_b[1:46])
    assert torch.equal(guard[1:2251].view(45, 50), ref_w) and torch.equal(guard_b[1:46], ref_b)
    assert bool((guard[2251:] == 7.0).all()) and bool((guard_b[46:] == 7.0).all()) and guard[0] == 7.0 and guard_b[0] == 7.0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TERMS))
@pytest.mark.parametrize("rows,outs", [(1, 1), (9000, 30), (40000, 3), (70, 1000)])
def test_bias_alone(dtype, rows, outs):
    """No columns: the bias gradient only, within rows * 2^-24 of the sum of magnitudes and a rounding to its type; added to what is
    there when asked."""
    dy = torch.randn(rows, outs, generator=torch.Generator().manual_seed(rows)).to(dtype).cuda()
    ck = ops.byte_store(torch.empty(rows, 0, dtype=dtype, device="cuda"))
    start = torch.randn(outs, generator=torch.Generator().manual_seed(2)).cuda()
    want = dy.double().cpu().sum(0)
    tol = rows * 2.0 ** -24 * dy.double().cpu().abs().sum(0) + 1e-37
    db = ops.byte_linear_grad(dy, ck, bias=True)[1]
    assert bool(((db.double().cpu() - want).abs() <= tol + ref.HALF_STEP[dtype] * (want.abs() + tol) + 2.0 ** -25).all())
    held = start.clone()
    ops.byte_linear_grad(dy, ck, out=torch.empty(outs, 0, device="cuda"), out_bias=held, accumulate=True)
    both = want + start.double().cpu()
    assert bool(((held.double().cpu() - both).abs() <= tol + 2.0 ** -23 * (both.abs() + tol)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TERMS))
def test_leading_dimensions_and_no_rows(dtype):
    x = torch.randn(3, 5, 40, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    dy = torch.randn(3, 5, 24, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    a, _ = ops.byte_linear_grad(dy, ops.byte_store(x))
    b, _ = ops.byte_linear_grad(dy.view(15, 24), ops.byte_store(x.view(15, 40)))
    assert torch.equal(a, b)
    dw, db = ops.byte_linear_grad(dy[:0], ops.byte_store(x[:0]), bias=True)
    assert not dw.any() and not db.any() and dw.shape == (24, 40)
    keep = torch.ones(24, 40, dtype=dtype, device="cuda")
    ops.byte_linear_grad(dy[:0], ops.byte_store(x[:0]), out=keep, accumulate=True)
    assert bool((keep == 1).all())
    dw, db = ops.byte_linear_grad(dy, ops.byte_store(x[..., :0]), bias=True)
    assert dw.shape == (24, 0) and torch.allclose(db.float(), dy.float().sum((0, 1)), rtol=2e-2, atol=1e-2)
    dw, _ = ops.byte_linear_grad(dy[..., :0], ops.byte_store(x))
    assert dw.shape == (0, 40)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(TERMS))
def test_what_is_not_finite_stays_in_its_row_or_column(dtype):
    rows, cols, outs = 70, 150, 140
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(5)).to(dtype).cuda()
    dy = torch.randn(rows, outs, generator=torch.Generator().manual_seed(6)).to(dtype).cuda()
    x[7, 31] = float("nan")
    x[8, 140] = -float("inf")                                   # held as NaN
    dy[9, 3] = float("nan")
    dy[10, 139] = float("inf")
    dw, db = ops.byte_linear_grad(dy, ops.byte_store(x), bias=True)
    bad = torch.zeros(outs, cols, dtype=torch.bool)
    bad[:, 31] = bad[:, 140] = True
    bad[3] = True
    assert torch.equal(torch.isnan(dw).cpu() | torch.isinf(dw).cpu(), bad | (torch.arange(outs) == 139)[:, None])
    held = ops.byte_load(ops.byte_store(x))
    fine = torch.isfinite(held).all(0)
    want = torch.where(held[10] == 0, float("nan"), torch.copysign(torch.full_like(held[10], float("inf")), held[10]))
    assert torch.equal(torch.nan_to_num(dw[139][fine].float(), nan=5.0), torch.nan_to_num(want[fine].float(), nan=5.0))
    assert torch.isnan(db[3]) and db[139] == float("inf") and int((~torch.isfinite(db)).sum()) == 2


@pytest.mark.gpu
def test_fp32_keeps_all_bits_of_dy():
    """One row: a product of a value of 24 bits and one of seven is rounded once."""
    dy = torch.randn(1, 300, generator=torch.Generator().manual_seed(8)).cuda()
    ck = ops.byte_store(torch.randn(1, 200, generator=torch.Generator().manual_seed(9)).cuda())
    dw, db = ops.byte_linear_grad(dy, ck, bias=True)
    want = dy.double().cpu().t() @ torch.from_numpy(ref.held(ck))
    assert bool(((dw.double().cpu() - want).abs() <= 4 * 2.0 ** -24 * want.abs()).all())   # three terms: three roundings and the last
    assert torch.equal(db, dy[0])


@pytest.mark.gpu
def test_refusals_on_the_gpu():
    ck, dy = _case(8, 40, 24, torch.bfloat16, "int8", 64)
    f = torch.zeros(24, 40, device="cuda")
    for call in (lambda: ops.byte_linear_grad(dy[:7], ck), lambda: ops.byte_linear_grad(dy.t(), ck), lambda: ops.byte_linear_grad(dy, ck, dtype=torch.float16),
                 lambda: ops.byte_linear_grad(dy, ck, accumulate=True), lambda: ops.byte_linear_grad(dy, ck, out=f.t()),
                 lambda: ops.byte_linear_grad(dy, ck, out=f[:, :39]), lambda: ops.byte_linear_grad(dy, ck, out=f, bias=True, accumulate=True),
                 lambda: ops.byte_linear_grad(dy, ck, out=f, out_bias=torch.zeros(24, device="cuda").bfloat16()),
                 lambda: ops.byte_linear_grad(dy.cpu(), ck), lambda: ops.byte_linear_grad(dy.double(), ck),
                 lambda: ops.byte_linear_grad(dy, ck, out=f, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("rows,cols,outs", [(64, 2 ** 31 - 1, 2 ** 31 - 1), (64, 2 ** 24 + 1, 8), (1000, 2 ** 31 - 1, 64), (10 ** 6, 2 ** 20, 2 ** 20),
                                            (64, 64, 2 ** 31 - 1), (64, 2 ** 12, 2 ** 24 + 64), (0, 2 ** 31 - 1, 2 ** 31 - 1)])
def test_no_workspace_for_sizes_that_are_refused(rows, cols, outs):
    """The query knows the limits of the call: no plan is made for a product that is refused."""
    s, P = binding.cmp_byte_shape(rows, cols, 0, 64), 4096
    assert binding.cmp_byte_linear_grad_work(s, outs, 0) == 0
    assert binding.cmp_byte_linear_grad(0, s, P, 1 << 62, P, 0, outs, outs, P, None, 0, False, P, 1 << 62, 0) == binding.CMP_E_ARG


def test_the_largest_products_have_a_plan():
    for cols, outs in ((2 ** 24, 2 ** 12), (2 ** 12, 2 ** 24), (2 ** 24, 8), (1, 2 ** 24), (2 ** 18 + 1, 2 ** 17 + 2 ** 16)):
        for rows in (0, 1, 2 ** 31 - 1):
            for kind in (0, 1, 2):
                assert binding.cmp_byte_linear_grad_work(binding.cmp_byte_shape(rows, cols, 0, 32), outs, kind) < 2 ** 45


@pytest.mark.parametrize("rows,cols,outs", [(183177, 44, 401), (56113, 54, 574), (190837, 53, 166), (123784, 24, 512)])
def test_ranges_of_fp32_fill_the_chip_once(rows, cols, outs):
    """Three terms of dY leave a CU one workgroup of 64 x 64 results (96 KB of LDS each), 256 of them on the chip: the ranges of
    rows, counted by their partial sums of dW and db, are no more than that."""
    work = binding.cmp_byte_linear_grad_work(binding.cmp_byte_shape(rows, cols, 0, 64), outs, binding.CMP_TYPE_F)
    ranges, rest = divmod(work, 4 * outs * (cols + 1))
    assert rest == 0 and 2 <= ranges <= 256 // -(-outs // 64)
