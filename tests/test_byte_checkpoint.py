"""Byte checkpoints: the bytes of the store and the values of the load, against the definition in 64 bits.

Bar: every byte and every value equal; scales are powers of two, so nothing but the code is rounded.
"""
import ctypes as C

import numpy as np
import pytest
import torch

import byte_reference as ref
from paper_2011_09017_amd import binding, operators as ops

TYPES = [torch.float32, torch.float16, torch.bfloat16]


# ---- without a GPU -------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,cols,group", [(0, 5, 32), (1, 1, 128), (3, 16, 32), (7, 33, 32), (5, 129, 64), (2, 0, 64)])
def test_sizes(rows, cols, group):
    n = binding.cmp_byte_bytes(binding.cmp_byte_shape(rows, cols, 0, group))
    pitch = -(-cols // 16) * 16
    assert n == -(-(rows * (pitch + -(-cols // group))) // 16) * 16


def test_library_refusals():
    """Bad arguments are refused before a device is touched (the pointers here are not memory)."""
    b, P = binding, 4096
    good = dict(rows=4, cols=40, format=0, group=32)
    n = b.cmp_byte_bytes(b.cmp_byte_shape(**good))
    assert n > 0
    for bad in (dict(group=16), dict(group=0), dict(group=96), dict(format=2), dict(rows=1 << 31), dict(cols=1 << 31)):
        s = b.cmp_byte_shape(**{**good, **bad})
        assert b.cmp_byte_bytes(s) == 0
        assert b.cmp_byte_store(0, s, P, 0, 1 << 32, P, 1 << 40, 0) == b.CMP_E_ARG
        assert b.cmp_byte_load(0, s, P, 1 << 40, P, 0, 1 << 32, 0) == b.CMP_E_ARG
        assert b.cmp_byte_linear_grad(0, s, P, 1 << 40, P, 0, 8, 8, P, None, 0, False, P, 1 << 40, 0) == b.CMP_E_ARG
    s = b.cmp_byte_shape(**good)
    for kw in (dict(x=0), dict(x=P + 2), dict(type=3), dict(ld=39), dict(ck=P + 8), dict(ck=0)):
        a = {**dict(x=P, type=0, ld=40, ck=P), **kw}
        assert b.cmp_byte_store(0, s, a["x"], a["type"], a["ld"], a["ck"], n, 0) == b.CMP_E_ARG, kw
        assert b.cmp_byte_load(0, s, a["ck"], n, a["x"], a["type"], a["ld"], 0) == b.CMP_E_ARG, kw
    assert b.cmp_byte_store(0, s, P, 0, 40, P, n - 1, 0) == b.CMP_E_NOSPACE
    assert b.cmp_byte_load(0, s, P, n - 1, P, 0, 40, 0) == b.CMP_E_FORMAT
    assert b.lib().cmp_byte_bytes(None) == 0
    assert b.lib().cmp_byte_store(0, None, P, 0, 40, P, n, 0) == b.CMP_E_ARG
    for device in (-1, 4097):
        assert b.cmp_byte_store(device, s, P, 0, 40, P, n, 0) in (b.CMP_E_ARG, b.CMP_E_HIP)


def test_python_refusals():
    x = torch.zeros(4, 40)
    for call in (lambda: ops.byte_store(x), lambda: ops.byte_store(x.int()), lambda: ops.byte_store(x.double()),
                 lambda: ops.byte_store(torch.tensor(1.0)), lambda: ops.byte_store(x, "int4"), lambda: ops.byte_store(x, group=48),
                 lambda: ops.byte_store(x.t()), lambda: ops.byte_store(torch.zeros(4, 8, 40)[:, :5]),
                 lambda: ops.byte_load(ops.ByteCheckpoint(torch.zeros(256, dtype=torch.uint8), (4, 40), torch.float32)),
                 lambda: ops.byte_load(ops.ByteCheckpoint(torch.zeros(256), (4, 40), torch.float32)),
                 lambda: ops.byte_load(ops.ByteCheckpoint(torch.zeros(256, dtype=torch.uint8), (4, 40), torch.float32, "int4"))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("make,want", [
    (lambda: torch.empty(3, 5, 8), (15, 8)), (lambda: torch.empty(3, 5, 8)[:, :, 1:6], (15, 8)), (lambda: torch.empty(3, 5, 8)[::2], None),
    (lambda: torch.empty(4, 5, 8)[:, 0], (4, 40)), (lambda: torch.empty(4, 5, 8)[:, :2], None), (lambda: torch.empty(8, 6).t(), None),
    (lambda: torch.empty(9), (1, 9)), (lambda: torch.empty(9)[::2], None), (lambda: torch.empty(1, 9)[:, 2:5], (1, 3)),
    (lambda: torch.empty(1, 7).expand(5, 7), None), (lambda: torch.empty(5, 1).expand(5, 1), (5, 1)), (lambda: torch.empty(0, 4), (0, 4)),
    (lambda: torch.empty(4, 0), (4, 0)), (lambda: torch.empty(6, 3)[:, 1:2], (6, 3)), (lambda: torch.empty(2, 1, 6, 4)[:, :, 2:, :3], None),
])
def test_rows_of_a_tensor(make, want):
    assert ops._rows_of(make()) == want


def test_reference_rounds_e4m3_like_torch():
    v = np.concatenate([np.linspace(0, 448, 20001), ref.e4m3_values(), (ref.e4m3_values()[1:] + ref.e4m3_values()[:-1]) / 2])
    got = ref.e4m3_values()[ref._nearest_even(v, ref.e4m3_values())]
    assert np.array_equal(got, torch.from_numpy(v).float().to(torch.float8_e4m3fn).double().numpy())


# ---- on the GPU ----------------------------------------------------------------------------------------
def _check(x, ck, rows, cols):
    codes, pad, exps, tail = ref.split(ck.buf.cpu().numpy(), rows, cols, ck.group)
    want_codes, want_exps = ref.encode(x.detach().double().cpu().reshape(rows, cols).numpy(), ck.fmt, ck.group)
    assert np.array_equal(exps, want_exps)
    if ck.fmt == "e4m3":                                      # the sign of a NaN is not stated
        codes = np.where((codes & 0x7f) == 0x7f, 0x7f, codes)
    assert np.array_equal(codes, want_codes)
    assert not pad.any() and not tail.any()
    return ref.decode(want_codes, want_exps, ck.fmt, ck.group)


def _same(y, want):
    want = torch.from_numpy(want).to(y.dtype) if y.dtype != torch.float16 else \
        torch.from_numpy(np.where(np.abs(want) > 65504, np.copysign(65504.0, want), want)).half()
    got = y.detach().cpu().reshape(want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got.float(), nan=0.0), torch.nan_to_num(want.float(), nan=0.0))


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 1), (1, 4096), (3, 7), (5, 33), (17, 64), (2, 3, 96), (64, 1000), (257, 129), (40, 16), (2, 8191)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt,group", [("int8", 32), ("int8", 64), ("int8", 128), ("e4m3", 32), ("e4m3", 64), ("e4m3", 128)])
def test_store_and_load(shape, dtype, fmt, group):
    gen = torch.Generator().manual_seed(sum(shape) + group)
    x = (torch.randn(shape, generator=gen) * torch.exp(2 * torch.randn(shape[-1], generator=gen))).to(dtype).cuda()
    rows, cols = x.numel() // shape[-1], shape[-1]
    n = binding.cmp_byte_bytes(binding.cmp_byte_shape(rows, cols, 0, group))
    buf = torch.full((n + 64,), 0xCD, dtype=torch.uint8, device="cuda")
    ck = ops.byte_store(x, fmt, group, out=buf)
    want = _check(x, ck, rows, cols)
    assert bool((buf[n:] == 0xCD).all())                       # nothing behind the checkpoint
    y = ops.byte_load(ck)
    assert y.shape == x.shape and y.dtype == dtype
    _same(y, want)
    for other in TYPES:
        _same(ops.byte_load(ck, dtype=other), want)


def _special(dtype):
    big = torch.finfo(dtype).max
    tiny = torch.finfo(dtype).tiny
    return [
        [0.0] * 40, [-0.0, 1.0, -1.0], [float("nan"), 1.0, 2.0], [float("inf"), 1.0, -float("inf")], [float("nan")] * 3,
        [float("inf")], [big, -big, big / 2, 1.0], [tiny, -tiny, tiny / 2, tiny * 64], [127.5, 0.5, 1.5, 2.5, -0.5, -127.5],
        [127.0, 63.5, 126.5], [128.0, 127.5, 0.75, 0.25], [448.0, 0.0009765625, 0.0029296875, -448.0], [464.0, 449.0, 2.0],
        [1.9921875, 1.0], [1.9922, 1.0], [1e-30, 1e-33], [2.0 ** -110, 2.0 ** -111, 2.0 ** -112], [3e4, 1e-4, 65504.0],
    ]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_special_values(dtype, fmt):
    """Zeros, ties, the borders of the exponent rule, the type's limits, NaN and infinities beside finite values."""
    rows = _special(dtype)
    x = torch.zeros(len(rows), 70)
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r)
        x[i, 66] = torch.tensor(r[-1])                           # a second group whose largest value is another
    x = x.to(dtype).cuda()
    ck = ops.byte_store(x, fmt, 64)
    _same(ops.byte_load(ck), _check(x, ck, len(rows), 70))
    # finite values beside a NaN keep their scale; the largest of the type does not overflow
    y = ops.byte_load(ck)
    assert torch.isfinite(y[torch.isfinite(x)]).all() and torch.isnan(y[~torch.isfinite(x)]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_strided_and_unaligned(dtype):
    """Rows further apart than they are long, bases off any alignment; nothing between the rows is read into a group or
    written by the load."""
    big = torch.full((50, 130), float("inf"), dtype=dtype, device="cuda")
    for lo, hi in ((1, 98), (3, 20), (0, 129), (5, 6)):
        x = big[:, lo:hi]
        vals = torch.randn(50, hi - lo, generator=torch.Generator().manual_seed(lo)).to(dtype).cuda()
        x.copy_(vals)
        ck = ops.byte_store(x, "int8", 32)
        want = _check(vals, ck, 50, hi - lo)
        out = torch.full((50, 130), 7.0, dtype=dtype, device="cuda")
        ops.byte_load(ck, out=out[:, lo:hi])
        _same(out[:, lo:hi], want)
        assert bool((out[:, :lo] == 7.0).all()) and bool((out[:, hi:] == 7.0).all())
        big[:, lo:hi] = float("inf")


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(0, 5), (5, 0), (0,), (2, 0, 3)])
def test_empty(shape):
    x = torch.zeros(shape, device="cuda")
    y = ops.byte_load(ops.byte_store(x))
    assert y.shape == x.shape


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A checkpoint of more than 2^32 bytes: the last rows."""
    rows, cols = 70001, 65536
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    last = torch.randn(3, cols, generator=torch.Generator().manual_seed(1)).bfloat16()
    x[-3:] = last.cuda()
    ck = ops.byte_store(x, "int8", 128)
    del x
    c, e = ref.encode(last.double().numpy(), "int8", 128)
    assert np.array_equal(ck.buf[rows * cols - 3 * cols:rows * cols].cpu().numpy().reshape(3, cols), c)
    y = ops.byte_load(ck)
    _same(y[-3:], ref.decode(c, e, "int8", 128))
    assert not y[:-3].any()


@pytest.mark.gpu
def test_refusals_on_the_gpu():
    x = torch.zeros(4, 40, device="cuda")
    ck = ops.byte_store(x)
    for call in (lambda: ops.byte_store(x, out=torch.zeros(256, device="cuda")), lambda: ops.byte_load(ck, out=x[:, :39]),
                 lambda: ops.byte_load(ck, dtype=torch.float64), lambda: ops.byte_load(ck, dtype=torch.float16, out=x),
                 lambda: ops.byte_store(x, out=torch.zeros(256, dtype=torch.uint8)),
                 lambda: ops.byte_load(ck, out=torch.zeros(40, 4, device="cuda").t())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(binding.CmpError) as e:
        ops.byte_store(x, out=torch.zeros(64, dtype=torch.uint8, device="cuda"))
    assert e.value.code == binding.CMP_E_NOSPACE
    with pytest.raises(binding.CmpError) as e:
        ops.byte_load(ck._replace(buf=ck.buf[:64]))
    assert e.value.code == binding.CMP_E_FORMAT
    with pytest.raises(binding.CmpError) as e:
        ops.byte_load(ck._replace(buf=torch.zeros(512, dtype=torch.uint8, device="cuda")[8:]))
    assert e.value.code == binding.CMP_E_ARG
