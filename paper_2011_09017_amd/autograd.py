"""Activation compression around autograd's saved tensors (phase 4 of the framework, Section 4.4).

The forward pass of a convolutional layer saves its input for the backward pass.  With the hooks
of this module installed, every saved fp32 NCHW activation is replaced by its compressed
container as soon as it is saved (``cmp_arena_push``) and restored when the backward pass asks for
it (``cmp_arena_pop``; data flow of Section 2.1).  The containers live in one device buffer that is
used as a stack: the backward pass consumes activations in the reverse order of the forward pass,
so the memory held at any time is the sum of the containers of the layers not yet differentiated.
Where each container lies is known to the GPU only (it depends on the sizes of those before it),
so neither hook ever waits for the GPU: compression runs behind the forward pass.

Nothing here computes: both hooks marshal arguments for the C ABI.  Parameters, tensors that are
not fp32 4-D CUDA tensors, small tensors and shapes the stack does not take are saved as they are.

What that codec does not take or does not shrink (bf16 and fp16, dense activations, channels last) can be held with
eight bits per value instead: :class:`ByteCheckpoints` are hooks of the same kind over byte checkpoints, and
:func:`linear` and :func:`group_norm` are layers whose backward pass reads the eight-bit form itself.  All of these can be
captured into a graph; as with any layer of torch, no eager graph of the same parameters may be alive while
``backward()`` is captured.
"""
from __future__ import annotations

import math
import re
import weakref
from dataclasses import dataclass
from typing import Callable, Iterable, Optional, Union

import torch
from torch.multiprocessing.reductions import StorageWeakRef

from . import binding, operators


class SlotStack:
    """Host mirror of the slot numbering of the device-side stack: slots are numbered in push order,
    and a number is free again once that slot and every slot above it have been released (exact
    for the forward/backward pattern; a release out of order leaves a hole until then)."""

    def __init__(self, capacity: int):
        self.capacity = int(capacity)
        self._live = []

    def push(self) -> int:
        if len(self._live) >= self.capacity:
            raise MemoryError(f"activation stack: more than {self.capacity} tensors held")
        self._live.append(True)
        return len(self._live) - 1

    def release(self, slot: int) -> None:
        if not (0 <= slot < len(self._live)) or not self._live[slot]:
            raise KeyError(slot)
        self._live[slot] = False
        while self._live and not self._live[-1]:
            self._live.pop()

    @property
    def held(self) -> int:
        return len(self._live)


@dataclass
class _Packed:
    """What autograd holds instead of the activation."""
    slot: int
    shape: tuple
    eb: float
    users: int = 1                              # one tensor may be saved by several nodes
    restored: Optional[torch.Tensor] = None     # kept between the first and the last unpack


class ActivationCompressor:
    """saved_tensors_hooks that compress activations.

    eb: the absolute error bound, or a callable ``eb(tensor) -> float`` (the adaptive
        controller of Sections 4.1-4.3 plugs in here).
    arena_bytes: capacity of the container stack on the GPU.
    max_numel: largest activation that will be compressed (sizes the context's scratch).
    min_numel: tensors smaller than this are saved uncompressed.
    slots: most activations held at once.
    """

    def __init__(self, eb: Union[float, Callable[[torch.Tensor], float]], arena_bytes: int, max_numel: int,
                 sub: int = 32, min_numel: int = 1 << 14, device: int = 0, slots: int = 1024):
        self.eb = eb
        self.min_numel = int(min_numel)
        self.max_numel = int(max_numel)
        self.device = torch.device("cuda", device)
        self.ctx = binding.Context(sub=sub, max_numel=self.max_numel, device=device)
        self.capacity = int(arena_bytes) // 256 * 256
        self.buffer = torch.empty(self.capacity, dtype=torch.uint8, device=self.device)
        self.state = torch.empty(binding.cmp_arena_state_bytes(slots), dtype=torch.uint8, device=self.device)
        self.stack = SlotStack(slots)
        rc = binding.cmp_arena_init(self.ctx._h, self.state.data_ptr(), slots, self._stream())
        if rc != binding.CMP_OK:
            raise binding.CmpError(rc, "cmp_arena_init")
        self._skip = set()                      # data pointers never to compress (parameters)
        self._by_tensor = {}                    # (data_ptr, version, shape) -> (weak ref, _Packed), current forward pass
        self.stats = {"packed": 0, "raw_bytes": 0, "passed_through": 0}
        self.on_unpack: Optional[Callable[[_Packed, torch.Tensor], None]] = None    # for tests

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def skip_parameters(self, params: Iterable[torch.Tensor]) -> None:
        for p in params:
            self._skip.add(p.data_ptr())

    # -- hooks -------------------------------------------------------------------------------
    def _wanted(self, t: torch.Tensor) -> bool:
        return (t.is_cuda and t.dtype == torch.float32 and t.dim() == 4 and t.is_contiguous()
                and self.min_numel <= t.numel() <= self.max_numel
                and not isinstance(t, torch.nn.Parameter) and t.data_ptr() not in self._skip
                and binding.cmp_arena_accepts(self.ctx._h, t.shape))

    def pack(self, t: torch.Tensor):
        if not self._wanted(t):
            self.stats["passed_through"] += 1
            return t
        # a tensor saved by several nodes (a ReLU output that is also the next convolution's input)
        # is compressed once; the weak reference tells a live tensor from a recycled address
        key = (t.data_ptr(), t._version, tuple(t.shape))
        hit = self._by_tensor.get(key)
        if hit is not None and hit[0]() is t:
            hit[1].users += 1
            return hit[1]
        eb = float(self.eb(t)) if callable(self.eb) else float(self.eb)
        slot = self.stack.push()
        rc = binding.cmp_arena_push(self.ctx._h, self.buffer.data_ptr(), self.capacity, self.state.data_ptr(), slot,
                                    t.data_ptr(), t.shape, eb, self._stream())        # does not wait
        if rc != binding.CMP_OK:
            self.stack.release(slot)
            raise binding.CmpError(rc, "cmp_arena_push")
        p = _Packed(slot, tuple(t.shape), eb)
        self._by_tensor[key] = (weakref.ref(t), p)
        self.stats["packed"] += 1
        self.stats["raw_bytes"] += 4 * t.numel()
        return p

    def unpack(self, p):
        if not isinstance(p, _Packed):
            return p
        if p.users <= 0:
            # the slot went back when the first saving node took its tensor and the last one
            # dropped it: a second backward over the same graph would read whatever lies there now
            raise RuntimeError("compressed activation already released: a graph whose saved tensors "
                               "were compressed can be walked backward once")
        if p.restored is None:
            out = torch.empty(p.shape, dtype=torch.float32, device=self.device)
            rc = binding.cmp_arena_pop(self.ctx._h, self.buffer.data_ptr(), self.state.data_ptr(), p.slot, p.shape,
                                       p.eb, out.data_ptr(), self._stream())          # decompresses, frees the slot
            if rc != binding.CMP_OK:
                raise binding.CmpError(rc, "cmp_arena_pop")
            self.stack.release(p.slot)
            p.restored = out
            if self.on_unpack is not None:
                self.on_unpack(p, p.restored)
        out = p.restored
        p.users -= 1
        if p.users == 0:
            p.restored = None
        return out

    def hooks(self):
        """Context manager for one forward pass: ``with compressor.hooks(): loss = model(x)``."""
        self._by_tensor = {}
        return torch.autograd.graph.saved_tensors_hooks(self.pack, self.unpack)

    def check(self) -> dict:
        """Waits for the GPU.  Raises if a push did not fit or a pop met a damaged container;
        returns the stack's figures: bytes in use, their peak, slots held, and the status of the
        calls so far (CMP_W_RANGE: some activation lay outside the quantiser's range and was clamped)."""
        rc, top, peak, held, failed = binding.cmp_arena_stats(self.ctx._h, self.state.data_ptr(), self._stream())
        st = self.ctx.last_status()
        if failed:
            raise MemoryError(f"activation stack: {failed} container(s) did not fit into {self.capacity} bytes")
        if st < 0:
            raise binding.CmpError(st, "activation stack")
        return {"top": top, "peak": peak, "held": held, "status": st}


# A parameter reaches an operation as it is, as a view of it, or as a copy of either in another type or order.
_FORMS_OF_A_PARAMETER = re.compile(r"(ToCopy|Clone|T|Transpose|Permute|View|UnsafeView|ReshapeAlias|Select|Slice|Split|SplitWithSizes|Unbind|"
                                   r"Expand|Squeeze|Unsqueeze|Alias|AsStrided)Backward\d*")


def _storage(t: torch.Tensor) -> int:
    return t.untyped_storage().data_ptr()


def _in_autocast() -> bool:
    # torch.is_autocast_enabled says no inside the operation whose arguments autocast has cast, which is where hooks run
    depth = torch.autocast_increment_nesting()
    torch.autocast_decrement_nesting()
    return depth > 1


@dataclass
class _HeldBytes:
    """What autograd holds instead of a tensor: its checkpoint in the order of its memory, and that order."""
    ck: operators.ByteCheckpoint
    order: tuple


class ByteCheckpoints:
    """saved_tensors_hooks that hold every saved fp32, fp16 or bf16 tensor as a byte checkpoint, whatever its shape and
    whatever the order of its dimensions in memory (channels last included; groups run along the dimension that is
    dense).  A graph can be walked backward as often as autograd allows: checkpoints are only read.  What several
    operations of a forward pass save (the input of three projections) is held once, as autograd itself has it (changes in
    between that torch does not count, through raw pointers, are not seen).

    fmt, group: see operators.byte_store.  min_numel: smaller tensors are saved as they are, and so are parameters
    (torch.nn.Parameter, frozen ones too), tensors named to skip_parameters, views of either and copies of them in another type or
    order (autocast's among them), tensors with gaps and those whose rows are too short for eight bits to save anything (a
    row of codes takes a multiple of 16 bytes).  Inside an autocast region tensors of its type without a gradient history are saved as
    they are too: a cast of a frozen weight looks like that.  Weights that are computed in another way (the sum of a weight
    and its low-rank change, a frozen one cast by the program) look like activations and have to be named.

    A value is off by at most 1/127 of the largest in its group ("int8") or 1/16 of itself ("e4m3"): what is not an activation
    (indices kept as floats, running sums, statistics that a layer keeps for its backward pass) does not belong under these hooks.
    """

    def __init__(self, fmt: str = "int8", group: int = 64, min_numel: int = 1 << 14):
        operators._byte_shape(0, 0, fmt, group)                       # refuses what byte_store would refuse later
        self.fmt, self.group, self.min_numel = fmt, int(group), int(min_numel)
        self._named = []                        # weak references: an address means what was named as long as that lives
        self._skip = set()                      # their storages
        self._by_memory = {}                    # what memory held -> (weak ref of its storage, of its checkpoint's bytes), current forward pass
        self.stats = {"packed": 0, "shared": 0, "raw_bytes": 0, "held_bytes": 0, "passed_through": 0}

    def skip_parameters(self, params: Iterable[torch.Tensor]) -> None:
        # of the tensor, whose storage may change, and of the storage, which outlives a view that only served to name it
        self._named += [(weakref.ref(p), StorageWeakRef(p.untyped_storage()), _storage(p)) for p in params]
        self._find_named()

    def _find_named(self) -> None:
        self._named = [n for n in self._named if n[0]() is not None or not n[1].expired()]
        tensors = [n[0]() for n in self._named]
        self._skip = {_storage(t) for t in tensors if t is not None} | {at for _, storage, at in self._named if not storage.expired()}

    def _is_weight(self, t: torch.Tensor) -> bool:
        def known(v):
            return isinstance(v, torch.nn.Parameter) or _storage(v) in self._skip
        base = t if t._base is None else t._base
        if known(base):
            return True
        node = base.grad_fn
        while node is not None and _FORMS_OF_A_PARAMETER.fullmatch(node.name()):
            node = node.next_functions[0][0]
        if hasattr(node, "variable"):                                 # a leaf: the tensor that accumulates a gradient
            return known(node.variable)
        return not t.requires_grad and t.dtype == torch.get_autocast_dtype(t.device.type) and _in_autocast()

    def _held_bytes(self, t: torch.Tensor, order: tuple) -> int:
        cols = t.shape[order[-1]]
        return operators._byte_shape(t.numel() // cols, cols, self.fmt, self.group)[1]

    def pack(self, t: torch.Tensor):
        if (not t.is_cuda or t.layout != torch.strided or t.dtype not in operators._TYPES or t.dim() < 1
                or t.numel() < max(1, self.min_numel) or self._is_weight(t)):
            self.stats["passed_through"] += 1
            return t
        # dimensions of one element last in the order of memory would make rows of one value: they come first
        order = tuple(sorted(range(t.dim()), key=lambda d: (t.shape[d] != 1, -t.stride(d), d)))
        if not t.permute(order).is_contiguous() or self._held_bytes(t, order) >= t.numel() * t.element_size():
            self.stats["passed_through"] += 1
            return t
        # Saved before and not changed since: the checkpoint of the same dense rows, whatever their shape (a layer of matrices saves a
        # view of its own).  The weak references tell live memory from recycled addresses and bytes in use from freed
        # ones; another stream has nothing to wait for the first one's store with, and a graph's replays do not repeat a store that was not captured.
        rows = t.detach().permute(order)
        storage = t.untyped_storage()
        key = (storage._cdata, t.storage_offset(), t.numel(), rows.shape[-1], t.dtype, t._version, operators._stream(t.device),
               torch.cuda.is_current_stream_capturing())
        hit = self._by_memory.get(key)
        buf = None if hit is None or hit[0].expired() else hit[1]()
        if buf is not None:
            self.stats["shared"] += 1
            return _HeldBytes(operators.ByteCheckpoint(buf, tuple(rows.shape), t.dtype, self.fmt, self.group), order)
        ck = operators.byte_store(rows, self.fmt, self.group)
        self._by_memory[key] = (StorageWeakRef(storage), weakref.ref(ck.buf))
        self.stats["packed"] += 1
        self.stats["raw_bytes"] += t.numel() * t.element_size()
        self.stats["held_bytes"] += ck.nbytes
        return _HeldBytes(ck, order)

    def unpack(self, h):
        if not isinstance(h, _HeldBytes):
            return h
        back = [0] * len(h.order)
        for i, d in enumerate(h.order):
            back[d] = i
        return operators.byte_load(h.ck).permute(back)

    def hooks(self):
        """Context manager for one forward pass: ``with held.hooks(): loss = model(x)``."""
        self._find_named()
        self._by_memory = {}
        return torch.autograd.graph.saved_tensors_hooks(self.pack, self.unpack)


def _dense_rows(t: torch.Tensor) -> torch.Tensor:
    """t, or a copy where its rows are not evenly spaced (the gradient of a sum comes as one expanded value)."""
    return t if operators._rows_of(t) is not None else t.contiguous()


def _as_matrix(t: torch.Tensor) -> torch.Tensor:
    return t.reshape(math.prod(t.shape[:-1]), t.shape[-1])


def _keep(ctx, held: Optional[operators.ByteCheckpoint], *tensors) -> None:
    """Saves tensors and a checkpoint for the backward pass; autograd frees its bytes with the others behind that pass."""
    ctx.held = None if held is None else held._replace(buf=None)
    ctx.save_for_backward(*tensors, None if held is None else held.buf)


def _kept(ctx):
    *tensors, buf = ctx.saved_tensors
    return None if buf is None else ctx.held._replace(buf=buf), *tensors


def _product(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor]) -> torch.Tensor:
    """The linear layer of a matrix: with more dimensions torch may choose a batched product."""
    return torch.nn.functional.linear(_as_matrix(x), weight, bias).view(*x.shape[:-1], weight.shape[0])


class _Linear(torch.autograd.Function):
    @staticmethod
    @torch.amp.custom_fwd(device_type="cuda")
    def forward(ctx, x, weight, bias, fmt, group, held):
        rows = _dense_rows(x)
        if not ctx.needs_input_grad[1]:
            held = None
        elif held is None:
            held = operators.byte_store(rows, fmt, group)
        _keep(ctx, held, weight if ctx.needs_input_grad[0] else None)
        ctx.kinds = (x.dtype, weight.dtype, None if bias is None else bias.dtype)
        return _product(rows, weight, bias)

    @staticmethod
    @torch.autograd.function.once_differentiable
    @torch.amp.custom_bwd(device_type="cuda")
    def backward(ctx, dy):
        held, weight = _kept(ctx)
        dx = dw = db = None
        dy = _dense_rows(dy)
        if ctx.needs_input_grad[0]:
            dx = torch.mm(_as_matrix(dy), weight.to(dy.dtype)).to(ctx.kinds[0]).view(*dy.shape[:-1], weight.shape[1])
        with_bias = ctx.kinds[2] is not None and ctx.needs_input_grad[2]
        if ctx.needs_input_grad[1]:
            dtype = torch.float32 if ctx.kinds[1] == torch.float32 else dy.dtype
            dw, db = operators.byte_linear_grad(dy, held, bias=with_bias, dtype=dtype)
            dw = dw.to(ctx.kinds[1])
        elif with_bias:
            db = _as_matrix(dy).sum(0, dtype=torch.float32)
        if db is not None:
            db = db.to(ctx.kinds[2])
        return dx, dw, db, None, None, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, fmt: str = "int8", group: int = 64,
           held: Optional[operators.ByteCheckpoint] = None):
    """torch.nn.functional.linear whose input is held as a byte checkpoint; the weight's (and bias's) gradient is computed from
    the eight-bit form by operators.byte_linear_grad.  x: [..., cols] in float32, float16 or bfloat16 on a GPU.  held: x's
    checkpoint where there is one already (operators.byte_store(x), for several layers of one input): it is read in place of a new
    one, and fmt and group are its own.  Without a backward pass to come (torch.no_grad, or a weight that needs
    no gradient) nothing is stored."""
    operators._byte_shape(0, 0, fmt, group)                           # refuses a bad format in either case
    if held is not None:
        operators._refuse(not isinstance(held, operators.ByteCheckpoint) or tuple(held.shape) != tuple(x.shape),
                          "linear: held has to be the checkpoint of x")
        operators._refuse(held.nbytes < binding.cmp_byte_bytes(operators._held(held)), "linear: held is too short for its shape")
        operators._refuse(held.buf.device != x.device, "linear: held is on another GPU than x")
    if not torch.is_grad_enabled():
        return _product(x, weight, bias)
    return _Linear.apply(x, weight, bias, fmt, group, held)


def _norm_parameters(*params):
    """gamma and beta as the operators take them."""
    return tuple(None if p is None else p.float().contiguous() for p in params)


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, act, fmt, group):
        x = x.contiguous()
        w, b = _norm_parameters(weight, bias)
        save = fmt if any(ctx.needs_input_grad) else None
        y, stats, held = operators.group_norm(x, groups, w, b, eps, act, save=save, group=group)
        ctx.groups, ctx.act = groups, act
        _keep(ctx, held, weight, bias, stats, None if held is not None else x)    # the parameters as they are: hooks know them
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        held, weight, bias, stats, x = _kept(ctx)
        w, b = _norm_parameters(weight, bias)
        params = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx, dw, db = operators.group_norm_grad(dy.contiguous(), held if x is None else x, stats, ctx.groups, w, b, ctx.act,
                                               params=params)
        dw = dw.to(weight.dtype) if params and ctx.needs_input_grad[1] else None
        db = db.to(bias.dtype) if params and ctx.needs_input_grad[2] else None
        return dx if ctx.needs_input_grad[0] else None, dw, db, None, None, None, None, None


def group_norm(x: torch.Tensor, groups: int, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5, act: str = "none", fmt: Optional[str] = "int8", group: int = 64):
    """Group norm and activation of x[batch, ..., channels] (channels last: permute an NCHW tensor to NHWC first, which costs
    nothing for one in torch's channels_last format).  Its input is held as a byte checkpoint written in the same pass;
    fmt=None holds x itself.  Without a backward pass to come (torch.no_grad, or nothing that needs a gradient) nothing is stored."""
    if fmt is not None:
        operators._byte_shape(0, 0, fmt, group)                       # refuses a bad format in either case
    return _GroupNorm.apply(x, weight, bias, groups, eps, act, fmt if torch.is_grad_enabled() else None, group)
