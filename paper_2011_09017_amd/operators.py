"""Operators on activations held in eight bits, and group norm: torch tensors in, torch tensors out.

Next to the container codec of :mod:`.binding` (fp32 NCHW activations with zeros and smooth planes) these hold any
activation as a *byte checkpoint* and compute a layer's backward pass from it:

* :func:`byte_store`, :func:`byte_load` -- a tensor to its checkpoint and back;
* :func:`byte_linear_grad` -- weight and bias gradient of a linear layer from its input's checkpoint;
* :func:`group_norm`, :func:`group_norm_grad` -- group norm with an activation, channels last, whose input can be
  kept as a checkpoint in the same pass.

Formats, formulas, limits and error bounds are those of include/cmpz.h.  The functions run on the current stream of
their tensors' GPU (which need not be the current GPU), wait for nothing, and may be captured into a graph; outputs and
workspaces that the caller does not pass come from torch's allocator.  They know nothing of autograd but that what a caller
passes to be written counts as changed: gradients flow through :mod:`.autograd`'s functions.  Wrong arguments raise ValueError before anything is launched, what the library
refuses raises :class:`.binding.CmpError`.
"""
from __future__ import annotations

import math
from functools import lru_cache
from typing import NamedTuple, Optional

import torch

from . import binding

_TYPES = {torch.float32: binding.CMP_TYPE_F, torch.float16: binding.CMP_TYPE_H, torch.bfloat16: binding.CMP_TYPE_BF}
_FORMATS = {"int8": binding.CMP_BYTE_INT, "e4m3": binding.CMP_BYTE_FLOAT}
_ACTS = {"none": binding.CMP_ACT_NONE, "relu": binding.CMP_ACT_RELU, "silu": binding.CMP_ACT_SILU}
GROUPS = (32, 64, 128)


def _refuse(cond, text: str) -> None:
    if cond:
        raise ValueError(text)


def _type_of(t: torch.Tensor) -> int:
    _refuse(not isinstance(t, torch.Tensor) or t.dtype not in _TYPES, "a float32, float16 or bfloat16 tensor is wanted")
    return _TYPES[t.dtype]


def _on_gpu(first: torch.Tensor, *others) -> torch.device:
    dev = first.device
    for t in others:
        _refuse(t is not None and t.device != dev, "all tensors have to be on one GPU")
    _refuse(dev.type != "cuda", "tensors on a GPU are wanted (there is no CPU path)")
    return dev


def _stream(dev: torch.device) -> int:
    return torch._C._cuda_getCurrentRawStream(dev.index)          # the current stream's handle, without a Stream object


def _call(rc: int, where: str, *written) -> None:
    """`written`: tensors of the caller's that the call has changed, None among them."""
    if rc != binding.CMP_OK:
        raise binding.CmpError(rc, where)
    for t in written:
        if t is not None:
            torch.autograd.graph.increment_version(t)


def _rows_of(t: torch.Tensor):
    """(rows, row stride) of a tensor seen as a matrix of its last dimension, None if its strides do not allow it."""
    cols = t.shape[-1]
    if t.is_contiguous():
        return (t.numel() // cols if cols else math.prod(t.shape[:-1])), cols
    if t.numel() == 0:
        return math.prod(t.shape[:-1]), cols
    if t.stride(-1) != 1 and cols != 1:
        return None
    rows, ld = 1, 0
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if rows == 1:
            ld = stride
        elif stride != ld * rows:
            return None
        rows *= size
    if rows == 1:
        ld = cols
    return (rows, ld) if ld >= cols else None


def _matrix(t: torch.Tensor, what: str):
    _refuse(t.dim() < 1, f"{what}: at least one dimension is wanted")
    at = _rows_of(t)
    _refuse(at is None, f"{what}: the last dimension has to be dense and the rows evenly spaced (call .contiguous())")
    return at


@lru_cache(maxsize=4096)
def _byte_shape(rows: int, cols: int, fmt: str, group: int):
    """(the C shape, bytes of a checkpoint): depend on sizes only and are read only."""
    _refuse(fmt not in _FORMATS, f"format {fmt!r}: {' or '.join(_FORMATS)}")
    _refuse(group not in GROUPS, f"groups of {group}: 32, 64 or 128")
    shape = binding.cmp_byte_shape(rows, cols, _FORMATS[fmt], group)
    return shape, binding.cmp_byte_bytes(shape)


@lru_cache(maxsize=4096)
def _linear_work(rows: int, cols: int, fmt: str, group: int, outs: int, kind: int) -> int:
    return binding.cmp_byte_linear_grad_work(_byte_shape(rows, cols, fmt, group)[0], outs, kind)


class ByteCheckpoint(NamedTuple):
    """An activation held in eight bits: the bytes, and what is needed to read them."""
    buf: torch.Tensor          # uint8, cmp_byte_bytes of them at least
    shape: tuple               # of the tensor that was stored; its last dimension is that of the groups
    dtype: torch.dtype         # of the tensor that was stored
    fmt: str = "int8"          # "int8" or "e4m3"
    group: int = 64            # columns of a scale: 32, 64 or 128

    @property
    def cols(self) -> int:
        return int(self.shape[-1])

    @property
    def rows(self) -> int:
        return math.prod(self.shape[:-1])

    @property
    def nbytes(self) -> int:
        return self.buf.numel()


def _held(ck: ByteCheckpoint):
    """The C shape of a checkpoint; its buffer has to be on a GPU, dense bytes."""
    _refuse(ck.buf.dtype != torch.uint8 or not ck.buf.is_contiguous(), "checkpoint: a contiguous uint8 buffer is wanted")
    _refuse(len(ck.shape) < 1, "checkpoint: at least one dimension is wanted")
    return _byte_shape(ck.rows, ck.cols, ck.fmt, ck.group)[0]


def byte_store(x: torch.Tensor, fmt: str = "int8", group: int = 64, out: Optional[torch.Tensor] = None) -> ByteCheckpoint:
    """Stores x (any shape, groups along the last dimension).  `out`: a uint8 buffer to store into, 16-byte aligned."""
    kind = _type_of(x)
    rows, ld = _matrix(x, "byte_store")
    shape, nbytes = _byte_shape(rows, x.shape[-1], fmt, group)
    dev = _on_gpu(x, out)
    given = out
    if out is None:
        out = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    _refuse(out.dtype != torch.uint8 or not out.is_contiguous(), "byte_store: out has to be a contiguous uint8 tensor")
    _call(binding.cmp_byte_store(dev.index, shape, x.data_ptr(), kind, ld, out.data_ptr(), out.numel(),
                                 _stream(dev)), "cmp_byte_store", given)
    return ByteCheckpoint(out, tuple(x.shape), x.dtype, fmt, group)


def byte_load(ck: ByteCheckpoint, dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Restores a checkpoint, in the type it was stored from unless `dtype` or `out` says otherwise."""
    shape = _held(ck)
    dev = _on_gpu(ck.buf, out)
    given = out
    if out is None:
        out = torch.empty(ck.shape, dtype=dtype or ck.dtype, device=dev)
    _refuse(tuple(out.shape) != tuple(ck.shape), "byte_load: out has another shape than the checkpoint")
    _refuse(dtype is not None and out.dtype != dtype, "byte_load: out has another type than dtype")
    kind = _type_of(out)
    rows, ld = _matrix(out, "byte_load")
    _call(binding.cmp_byte_load(dev.index, shape, ck.buf.data_ptr(), ck.buf.numel(), out.data_ptr(), kind, ld,
                                _stream(dev)), "cmp_byte_load", given)
    return out


def byte_linear_grad(dy: torch.Tensor, ck: ByteCheckpoint, bias: bool = False, dtype: Optional[torch.dtype] = None,
                     out: Optional[torch.Tensor] = None, out_bias: Optional[torch.Tensor] = None, accumulate: bool = False):
    """(dW, db) of y = x W^T + b from dy[..., outs] and the checkpoint of x[..., cols]; db is None unless `bias` or `out_bias`
    asks for it.  Results in dy's type, or float32 with dtype=torch.float32.  accumulate: adds to `out` (and `out_bias`)."""
    kind = _type_of(dy)
    rows, ld = _matrix(dy, "byte_linear_grad")
    shape = _held(ck)
    _refuse(rows != ck.rows, f"byte_linear_grad: dy has {rows} rows, the checkpoint {ck.rows}")
    dev = _on_gpu(dy, ck.buf, out, out_bias)
    outs, cols = int(dy.shape[-1]), ck.cols
    _refuse(accumulate and out is None, "byte_linear_grad: accumulate needs out")
    _refuse(accumulate and bias and out_bias is None, "byte_linear_grad: accumulate with a bias needs out_bias")
    _refuse(out is not None and dtype is not None and out.dtype != dtype, "byte_linear_grad: out has another type than dtype")
    given = out, out_bias
    dtype = out.dtype if out is not None else dtype or dy.dtype
    _refuse(dtype not in (dy.dtype, torch.float32), "byte_linear_grad: results are in dy's type or float32")
    if out is None:
        out = torch.empty(outs, cols, dtype=dtype, device=dev)
    if out_bias is None and bias:
        out_bias = torch.empty(outs, dtype=dtype, device=dev)
    _refuse(tuple(out.shape) != (outs, cols) or not out.is_contiguous(), "byte_linear_grad: out has to be contiguous, [outs, cols]")
    _refuse(out_bias is not None and (tuple(out_bias.shape) != (outs,) or not out_bias.is_contiguous() or out_bias.dtype != dtype),
            "byte_linear_grad: out_bias has to be [outs], contiguous, of out's type")
    need = _linear_work(rows, cols, ck.fmt, ck.group, outs, kind)
    work = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(binding.cmp_byte_linear_grad(dev.index, shape, ck.buf.data_ptr(), ck.buf.numel(), dy.data_ptr(), kind, outs, ld,
                                       out.data_ptr(), None if out_bias is None else out_bias.data_ptr(), _TYPES[dtype],
                                       accumulate, None if work is None else work.data_ptr(), need,
                                       _stream(dev)), "cmp_byte_linear_grad", *given)
    return out, out_bias


@lru_cache(maxsize=4096)
def _norm_plan(batch: int, spatial: int, channels: int, groups: int, kind: int, act: str, eps: float, backward: bool, part: int):
    """(the C shape, bytes of the workspace): depend on sizes only and are read only."""
    _refuse(not 0 <= groups < 1 << 32 or channels >= 1 << 32, f"group norm: {groups} groups of {channels} channels")   # fields of 32 bits
    _call(binding.CMP_E_ARG if groups > channels else binding.CMP_OK, "cmp_group_norm")     # before statistics of so many are allocated
    shape = binding.cmp_norm_shape(batch, spatial, channels, groups, kind, _ACTS[act], eps)
    return shape, (binding.cmp_group_norm_grad_work if backward else binding.cmp_group_norm_forward_work)(shape, part)


def _norm_shape(x: torch.Tensor, groups: int, eps: float, act: str, backward: bool, part: int):
    """part: forward the columns of a scale of the checkpoint, 0 without one; backward whether the parameters' gradients are wanted."""
    _refuse(act not in _ACTS, f"activation {act!r}: {', '.join(_ACTS)}")
    _refuse(x.dim() < 2, "group norm: [batch, ..., channels] is wanted")
    _refuse(not x.is_contiguous(), "group norm: a contiguous tensor is wanted, channels last")
    return _norm_plan(x.shape[0], math.prod(x.shape[1:-1]), x.shape[-1], groups, _type_of(x), act, eps, backward, part)


def _parameter(t: Optional[torch.Tensor], channels: int, what: str):
    if t is None:
        return None
    _refuse(t.dtype != torch.float32 or tuple(t.shape) != (channels,) or not t.is_contiguous(),
            f"group norm: {what} has to be float32, contiguous, one value per channel")
    return t.data_ptr()


def group_norm(x: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5, act: str = "none", save: Optional[str] = None, group: int = 64):
    """(y, stats, checkpoint) of x[batch, ..., channels]: y = act(group norm of x), act "none", "relu" or "silu"; stats is what
    :func:`group_norm_grad` needs; save="int8" or "e4m3" keeps x as a checkpoint (groups of `group` channels), else None."""
    _refuse(save is not None and group not in GROUPS, f"groups of {group}: 32, 64 or 128")
    shape, need = _norm_shape(x, groups, eps, act, False, group if save is not None else 0)
    dev = _on_gpu(x, weight, bias)
    gamma, beta = _parameter(weight, x.shape[-1], "weight"), _parameter(bias, x.shape[-1], "bias")
    y = torch.empty_like(x)
    stats = torch.empty(x.shape[0], groups, 2, dtype=torch.float64, device=dev)
    ck, fmt = None, 0
    if save is not None:
        held, nbytes = _byte_shape(shape.batch * shape.spatial, shape.channels, save, group)
        fmt = held.format
        ck = ByteCheckpoint(torch.empty(nbytes, dtype=torch.uint8, device=dev), tuple(x.shape), x.dtype, save, group)
    work = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(binding.cmp_group_norm_forward(dev.index, shape, x.data_ptr(), gamma, beta, y.data_ptr(), stats.data_ptr(), fmt, group,
                                         None if ck is None else ck.buf.data_ptr(), 0 if ck is None else ck.buf.numel(),
                                         None if work is None else work.data_ptr(), need, _stream(dev)), "cmp_group_norm")
    return y, stats, ck


def group_norm_grad(dy: torch.Tensor, x, stats: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None,
                    bias: Optional[torch.Tensor] = None, act: str = "none", params: bool = True):
    """(dx, dweight, dbias) from dy, the input (a tensor of dy's type, or its :class:`ByteCheckpoint`), and what the forward
    pass was called with and gave.  params=False: the last two are None."""
    shape, need = _norm_shape(dy, groups, 1.0, act, True, bool(params))   # eps is in stats
    held = isinstance(x, ByteCheckpoint)
    src = x.buf if held else x
    dev = _on_gpu(dy, src, stats, weight, bias)
    _refuse(tuple(x.shape) != tuple(dy.shape), "group_norm_grad: dy has another shape than the input")
    _refuse(not held and (x.dtype != dy.dtype or not x.is_contiguous()), "group_norm_grad: the input has to be contiguous, of dy's type")
    _refuse(stats.dtype != torch.float64 or tuple(stats.shape) != (dy.shape[0], groups, 2) or not stats.is_contiguous(),
            "group_norm_grad: stats as group_norm gave them are wanted")
    gamma, beta = _parameter(weight, dy.shape[-1], "weight"), _parameter(bias, dy.shape[-1], "bias")
    fmt, group = 0, 64
    if held:
        fmt, group = _held(x).format, x.group
    dx = torch.empty_like(dy)
    dweight = dbias = None
    if params:
        dweight, dbias = torch.empty(2, dy.shape[-1], dtype=torch.float32, device=dev).unbind(0)
    work = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(binding.cmp_group_norm_grad(dev.index, shape, dy.data_ptr(), None if held else x.data_ptr(), fmt, group,
                                      src.data_ptr() if held else None, src.numel() if held else 0, gamma, beta, stats.data_ptr(),
                                      dx.data_ptr(), dweight.data_ptr() if params else None, dbias.data_ptr() if params else None,
                                      None if work is None else work.data_ptr(), need, _stream(dev)), "cmp_group_norm_grad")
    return dx, dweight, dbias
