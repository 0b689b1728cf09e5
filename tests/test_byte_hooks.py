"""What the saved-tensor hooks over byte checkpoints take and what they leave: weights stay as they are, in every form in which
a layer saves them."""
import pytest
import torch
import torch.nn.functional as F

from paper_2011_09017_amd import operators as ops
from paper_2011_09017_amd.autograd import ByteCheckpoints

DEV = "cuda"


class _Recorder(ByteCheckpoints):
    """The hooks with a store that only notes what it was given, and a GPU that need not be there."""

    def __init__(self, **kw):
        super().__init__(min_numel=1, **kw)
        self.seen = []

    def pack(self, t):
        self.seen.append((tuple(t.shape), self._is_weight(t)))
        return t

    def taken(self):
        return sorted(shape for shape, weight in self.seen if not weight)

    def left(self):
        return sorted(shape for shape, weight in self.seen if weight)


def _linear(dtype=torch.float32, learns=True):
    return torch.nn.Linear(64, 48).to(dtype).requires_grad_(learns)


@pytest.mark.parametrize("autocast", ["none", "outside", "inside"])
@pytest.mark.parametrize("learns", [True, False])
@pytest.mark.parametrize("dims", [(10, 64), (2, 5, 64)])
def test_weights_of_linear_layers_are_known(autocast, learns, dims):
    """A linear layer saves its weight transposed, under autocast a cast copy of it; the input is an activation of a layer
    before, which has a history."""
    layer = _linear(learns=learns)
    x = torch.randn(dims, requires_grad=True)
    held = _Recorder()
    cast = torch.autocast("cpu", dtype=torch.bfloat16, enabled=autocast != "none")
    if autocast == "outside":
        with cast, held.hooks():
            y = layer(x.exp())
    else:
        with held.hooks(), cast:
            y = layer(x.exp())
    y.float().sum().backward()
    assert held.left() == [(64, 48)]
    assert (64, 48) not in held.taken() and len(held.taken()) == (2 if learns else 1)     # the exponential's result, the layer's input


@pytest.mark.parametrize("autocast", [False, True])
def test_weights_of_convolutions_are_known(autocast):
    conv = torch.nn.Conv2d(8, 16, 3)
    x = torch.randn(2, 8, 9, 9, requires_grad=True)
    held = _Recorder()
    with held.hooks(), torch.autocast("cpu", dtype=torch.bfloat16, enabled=autocast):
        conv(x.exp())
    assert held.left() == [(16, 8, 3, 3)] and held.taken() == [(2, 8, 9, 9)] * 2


def test_views_casts_and_copies_of_parameters_are_known():
    w = torch.nn.Parameter(torch.randn(48, 64))
    x = torch.randn(10, 64, requires_grad=True)
    for form in (lambda: w[:32], lambda: w.bfloat16(), lambda: w[:32].bfloat16(), lambda: w.clone(), lambda: w.t().contiguous().bfloat16().t(),
                 lambda: w.chunk(2)[1].half(), lambda: w.view(2, 24, 64)[1], lambda: w.reshape(64, 48).reshape(48, 64).double().float()):
        held = _Recorder()
        v = form()
        with held.hooks():
            F.linear(x.to(v.dtype), v)
        assert len(held.left()) == 1 and held.left()[0] == (64, v.shape[0]), form
        assert held.taken() == [(10, 64)]


def test_activations_are_not_taken_for_weights():
    """Casts and views of an activation, of a leaf that is no parameter, and what is computed from a parameter and an input."""
    w = torch.nn.Parameter(torch.randn(64))
    x = torch.randn(2, 5, 64, requires_grad=True)
    held = _Recorder()
    for v in (x, x.detach(), x.bfloat16(), x.view(10, 64).t(), x.exp(), x.exp().bfloat16().permute(1, 0, 2), x * w, (x * w).view(-1).clone(),
              x.detach() + w):
        assert not held._is_weight(v)


def test_what_is_named_is_known_by_its_storage():
    """A plain tensor used as a weight is named; views of it, casts of it and its new storage after a change are meant too."""
    w = torch.randn(48, 64, requires_grad=True)
    f = torch.randn(48, 64)
    held = _Recorder()
    held.skip_parameters([w, f])
    other = torch.randn(48, 64, requires_grad=True)
    for v in (w, w.t(), w[8:], w.bfloat16(), w[8:].t().half(), f, f[3:], f.t()):
        assert held._is_weight(v)
    assert not held._is_weight(other.t()) and not held._is_weight(other.bfloat16())
    w.data = torch.randn(48, 64)
    with held.hooks():                                            # a forward pass begins: addresses as they are now
        assert held._is_weight(w.detach()) and held._is_weight(f[3:])
    at = f.untyped_storage().data_ptr()
    del f, v
    with held.hooks():
        assert at not in held._skip


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("autocast", [False, True])
@pytest.mark.parametrize("dims", [(64, 256), (4, 16, 256)])
@pytest.mark.parametrize("learns", [True, False])
def test_input_gradient_of_a_linear_layer_is_the_plain_one(dtype, autocast, dims, learns):
    """256 x 192 weights, above the smallest size that is held; nothing is named.  dx is the same product either way."""
    torch.manual_seed(3)
    layer = torch.nn.Linear(256, 192).to(DEV, dtype).requires_grad_(learns)
    x = torch.randn(dims, device=DEV).to(dtype).requires_grad_()
    got = []
    for held in (ByteCheckpoints(min_numel=1 << 13), None):
        with torch.autocast(DEV, dtype=torch.bfloat16, enabled=autocast):
            if held is None:
                y = layer(x)
            else:
                with held.hooks():
                    y = layer(x)
        dy = torch.randn(y.shape, generator=torch.Generator().manual_seed(1)).to(DEV, y.dtype)
        got.append(torch.autograd.grad(y, x, dy)[0])
        if held is not None:
            assert held.stats["packed"] == (1 if learns else 0)   # the input alone
    assert torch.equal(*got)


@pytest.mark.gpu
@pytest.mark.parametrize("autocast", [False, True])
def test_a_convolution_holds_its_input_only(autocast, monkeypatch):
    conv = torch.nn.Conv2d(32, 64, 3).to(DEV, memory_format=torch.channels_last)
    x = torch.randn(4, 32, 24, 24, device=DEV).to(memory_format=torch.channels_last).requires_grad_()
    held = ByteCheckpoints(min_numel=1 << 13)
    with torch.autocast(DEV, dtype=torch.bfloat16, enabled=autocast), held.hooks():
        y = conv(x)
    assert held.stats["packed"] == 1 and held.stats["raw_bytes"] == x.numel() * (2 if autocast else 4)
    y.float().sum().backward()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_layers_own_parameters_stay_as_they_are(dtype):
    """The eight-bit layers under the hooks of the same kind: weight, gamma and beta are saved unchanged, of whatever type."""
    from paper_2011_09017_amd.autograd import group_norm, linear
    gen = torch.Generator().manual_seed(4)
    gamma, beta = (torch.nn.Parameter(torch.randn(64, generator=gen).to(DEV, dtype)) for _ in range(2))
    w = torch.nn.Parameter(torch.randn(48, 64, generator=gen).to(DEV, dtype))
    x = torch.randn(3, 40, 64, generator=gen).to(DEV, dtype).requires_grad_()
    dy = torch.randn(3, 40, 48, generator=gen).to(DEV, dtype)
    got = []
    for held in (ByteCheckpoints(min_numel=1), None):
        if held is None:
            y = linear(group_norm(x, 8, gamma, beta, act="silu"), w)
        else:
            with held.hooks():
                y = linear(group_norm(x, 8, gamma, beta, act="silu"), w)
            assert held.stats["packed"] == 0
        got.append(torch.autograd.grad(y, (x, gamma, beta, w), dy))
    for a, b in zip(*got):
        assert torch.equal(a, b)


def _input(dtype=torch.bfloat16, shape=(4, 32, 256), seed=5):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(DEV, dtype).requires_grad_()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(128, 256), (4, 32, 256)])
def test_what_several_layers_save_is_held_once(shape):
    """Three projections of one activation: one checkpoint, the gradients of three, and the memory back behind the backward
    pass although the hooks live on."""
    torch.manual_seed(6)
    layers = [torch.nn.Linear(256, 128).to(DEV, torch.bfloat16) for _ in range(3)]
    x = _input(shape=shape)
    held = ByteCheckpoints("int8", 64, min_numel=1 << 10)
    dy = torch.randn(*shape[:-1], 128, generator=torch.Generator().manual_seed(7)).to(DEV, torch.bfloat16)
    with held.hooks():
        h = x * 2                                                 # (saves nothing)
        ys = [layer(h) for layer in layers]
    one = 128 * (256 + 256 // 64)
    assert held.stats["packed"] == 1 and held.stats["shared"] == 2 and held.stats["held_bytes"] == one
    assert held.stats["raw_bytes"] == 2 * x.numel()
    got = torch.autograd.grad([y for y in ys], [layer.weight for layer in layers], [dy] * 3, retain_graph=True)
    again = torch.autograd.grad([y for y in ys], [layer.weight for layer in layers], [dy] * 3)
    x2 = ops.byte_load(ops.byte_store(h.detach().view(-1, 256), "int8", 64))
    for layer, g, a in zip(layers, got, again):
        want = torch.autograd.grad(layer(x2), layer.weight, dy.view(-1, 128))[0]
        assert torch.equal(g, want) and torch.equal(a, want)


@pytest.mark.gpu
def test_shared_bytes_are_freed_with_their_last_user():
    x = _input(shape=(512, 1024))
    w = [torch.nn.Parameter(torch.randn(8, 1024, device=DEV).bfloat16()) for _ in range(2)]
    held = ByteCheckpoints(min_numel=1 << 12)

    def step():
        with held.hooks():
            h = x * 2
            return sum(F.linear(h, v) for v in w).float().square().sum()
    step().backward()
    before = torch.cuda.memory_allocated()
    loss = step()
    assert torch.cuda.memory_allocated() >= before + 512 * 1024
    loss.backward()
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() < before + 512 * 1024
    assert held.stats["packed"] == 4 and held.stats["shared"] == 2   # two steps: h and the square's 512 x 8 values; h's second user


@pytest.mark.gpu
def test_what_changed_or_lies_elsewhere_is_not_shared():
    """The same memory after a change in place, another part of it, another last dimension, another type of its bytes, the
    same addresses after the tensor is gone, and another stream: each has a checkpoint of its own."""
    held = ByteCheckpoints("e4m3", 32, min_numel=1)
    values = lambda t: ops.byte_load(ops.byte_store(t.contiguous(), "e4m3", 32))  # noqa: E731
    with held.hooks():
        x = _input(shape=(64, 256)).detach()
        first = held.pack(x)
        want = values(x)
        assert torch.equal(held.unpack(held.pack(x.view(2, 32, 256))).view(64, 256), want) and held.stats["shared"] == 1
        assert torch.equal(held.unpack(held.pack(x.unsqueeze(1)))[:, 0], want) and held.stats["shared"] == 2
        turned = x.t()                                            # the same rows in memory, seen from the other side
        assert torch.equal(held.unpack(held.pack(turned)), want.t()) and held.stats["shared"] == 3
        for v in (x[:32], x[32:], x.view(32, 512), x.view(torch.float16)):
            assert torch.equal(held.unpack(held.pack(v)).nan_to_num(), values(v).nan_to_num())
        assert held.stats["shared"] == 3
        x.mul_(3)
        assert torch.equal(held.unpack(held.pack(x)), values(x)) and held.stats["shared"] == 3
        assert torch.equal(held.unpack(first), want)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = held.pack(x)
        torch.cuda.synchronize()
        assert held.stats["shared"] == 3 and torch.equal(held.unpack(other), values(x))
        kept = []
        for k in range(4):                                        # one address after the other
            t = torch.full((64, 256), float(k + 1), device=DEV, dtype=torch.bfloat16)
            kept.append(held.pack(t))
            del t
        assert held.stats["shared"] == 3
        for k, h in enumerate(kept):
            assert bool((held.unpack(h) == k + 1).all())
        n = held.stats["packed"]
        x2 = _input(shape=(64, 256)).detach()
        held.pack(x2)                                             # dropped at once: nothing to share
        held.pack(x2)
        assert held.stats["packed"] == n + 2


@pytest.mark.gpu
def test_a_buffer_written_by_an_operator_counts_as_changed():
    """A caller's buffer that an operator fills between two layers: each layer's checkpoint is of what it saw."""
    held = ByteCheckpoints("int8", 32, min_numel=1)
    a, b = (ops.byte_store(_input(shape=(64, 256), seed=s).detach()) for s in (8, 9))
    buf = torch.empty(64, 256, device=DEV, dtype=torch.bfloat16)
    with held.hooks():
        kept = [held.pack(ops.byte_load(ck, out=buf)) for ck in (a, b)]
    assert held.stats["shared"] == 0 and not torch.equal(held.unpack(kept[0]), held.unpack(kept[1]))
    outs = [torch.zeros(a.nbytes, dtype=torch.uint8, device=DEV), torch.zeros(8, 256, device=DEV), torch.zeros(8, device=DEV)]
    dy, before = torch.ones(64, 8, device=DEV), [t._version for t in outs]
    ops.byte_store(buf, "int8", 64, out=outs[0])
    ops.byte_linear_grad(dy, a, out=outs[1], out_bias=outs[2])
    assert [t._version for t in outs] == [v + 1 for v in before]


def test_linear_refuses_another_tensors_checkpoint():
    from paper_2011_09017_amd.autograd import linear
    x, w = torch.randn(3, 5, 32), torch.randn(7, 32, requires_grad=True)
    buf = torch.empty(15 * 33 + 1, dtype=torch.uint8)
    good = ops.ByteCheckpoint(buf, (3, 5, 32), torch.float32, "int8", 32)
    with torch.no_grad():
        assert torch.equal(linear(x, w, held=good), F.linear(x, w))
    for bad in (good._replace(shape=(15, 32)), good._replace(fmt="int4"), good._replace(group=48), good._replace(buf=buf.int()),
                good._replace(buf=buf[::2]), good._replace(buf=buf[:400]), buf, good._replace(buf=buf.to("meta"))):
        for grad in (True, False):
            with torch.set_grad_enabled(grad), pytest.raises(ValueError):
                linear(x, w, held=bad)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,group", [("int8", 64), ("e4m3", 128)])
def test_layers_of_one_input_share_a_checkpoint(fmt, group, monkeypatch):
    """Three projections of one activation from one checkpoint: what each gives with its own, and one checkpoint's memory."""
    from paper_2011_09017_amd.autograd import linear
    gen = torch.Generator().manual_seed(10)
    ws = [torch.nn.Parameter(torch.randn(n, 256, generator=gen).to(DEV, torch.bfloat16)) for n in (128, 64, 64)]
    bs = [torch.nn.Parameter(torch.randn(len(w), generator=gen).to(DEV, torch.bfloat16)) for w in ws]
    x = _input()
    dys = [torch.randn(4, 32, len(w), generator=gen).to(DEV, torch.bfloat16) for w in ws]
    want = torch.autograd.grad([linear(x, w, b, fmt, group) for w, b in zip(ws, bs)], [x, *ws, *bs], dys)
    stores = []
    real = ops.byte_store
    monkeypatch.setattr(ops, "byte_store", lambda *a, **kw: (stores.append(1), real(*a, **kw))[1])
    held = ops.byte_store(x.detach(), fmt, group)
    ys = [linear(x, w, b, held=held) for w, b in zip(ws, bs)]
    for a, b in zip(torch.autograd.grad(ys, [x, *ws, *bs], dys), want):
        assert torch.equal(a, b)
    assert len(stores) == 1


@pytest.mark.parametrize("learns", range(4))
def test_a_norm_that_nothing_learns_from_stores_nothing(learns, monkeypatch):
    """With gradients enabled a checkpoint is written if one of input, weight and bias needs one (0: none does)."""
    from paper_2011_09017_amd.autograd import group_norm
    asked = []

    def norm(x, groups, w, b, eps, act, save=None, group=64):
        asked.append(save)
        ck = None if save is None else ops.ByteCheckpoint(torch.empty(0, dtype=torch.uint8), tuple(x.shape), x.dtype, save, group)
        return torch.empty_like(x), torch.empty(x.shape[0], groups, 2, dtype=torch.float64), ck
    monkeypatch.setattr(ops, "group_norm", norm)
    ts = [torch.randn(s) for s in ((2, 9, 32), (32,), (32,))]
    if learns:
        ts[learns - 1].requires_grad_()
    y = group_norm(ts[0], 4, ts[1], ts[2], fmt="e4m3")
    assert asked == ["e4m3" if learns else None] and y.requires_grad == bool(learns)


@pytest.mark.gpu
def test_shared_checkpoints_replay_from_a_graph():
    """Three projections under the hooks and three with one checkpoint, forward and backward, captured once; every replay on
    changed inputs, with eager steps between, gives the eager results."""
    from paper_2011_09017_amd.autograd import linear
    gen = torch.Generator().manual_seed(11)
    ws = [torch.nn.Parameter(torch.randn(64, 256, generator=gen).to(DEV, torch.bfloat16)) for _ in range(3)]
    sets = [[torch.randn(4, 32, n, generator=gen).to(DEV, torch.bfloat16) for n in (256, 64)] for _ in range(3)]
    held = ByteCheckpoints("int8", 64, min_numel=1 << 10)

    def step(x, dy):
        x = x.detach().requires_grad_()
        with held.hooks():
            ys = [F.linear(x * 2, w) for w in ws[:1]] + [F.linear(x, w) for w in ws]
        ck = ops.byte_store(x.detach())
        ys += [linear(x, w, held=ck) for w in ws]
        return [y.detach() for y in ys] + list(torch.autograd.grad(ys, [x, *ws], [dy] * len(ys)))

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
    for v in (1, 2, 0, 1):
        for a, s in zip(ins, sets[v]):
            a.copy_(s)
        g.replay()
        torch.cuda.synchronize()
        for t, u in zip(outs, want[v]):
            assert torch.equal(t, u)
        step(*sets[(v + 1) % 3])
        torch.cuda.synchronize()


def test_names_given_by_a_temporary_last_as_long_as_their_memory():
    """A view or a detached alias that nobody keeps names the tensor behind it."""
    for alias in (lambda t: t.t(), lambda t: t.data, lambda t: t.detach()[3:], lambda t: t.view(-1)):
        w = torch.randn(48, 64)
        held = _Recorder()
        held.skip_parameters(alias(t) for t in [w])
        with held.hooks():
            assert held._is_weight(w) and held._is_weight(w.t())
        at = w.untyped_storage().data_ptr()
        del w
        with held.hooks():
            assert at not in held._skip
