"""The eight-bit layers as a network uses them: group norm, activation and linear layers in a row through autograd, the
saved-tensor hooks, graph capture, streams."""
import pytest
import torch

import byte_reference as ref
from paper_2011_09017_amd import operators as ops
from paper_2011_09017_amd.autograd import ByteCheckpoints, group_norm, linear

DEV = "cuda"


def test_hooks_refuse_and_pass_through_without_a_gpu():
    for kw in (dict(fmt="int4"), dict(group=48)):
        with pytest.raises(ValueError):
            ByteCheckpoints(**kw)
    held = ByteCheckpoints(min_numel=1)
    x = torch.randn(64, 64, requires_grad=True)
    with held.hooks():
        loss = (x * x).sum()
    loss.backward()                                              # tensors on the CPU stay as they are
    assert held.stats["packed"] == 0 and torch.equal(x.grad, 2 * x.detach())


def test_without_gradients_nothing_is_stored_and_formats_are_checked():
    x, w = torch.randn(3, 5, 32), torch.randn(7, 32, requires_grad=True)
    with torch.no_grad():
        assert torch.equal(linear(x, w), torch.nn.functional.linear(x, w))       # no GPU is needed where nothing is stored
        for layer in (lambda **kw: linear(x, w, **kw), lambda **kw: group_norm(x, 4, **kw)):
            for kw in (dict(fmt="int4"), dict(group=48)):
                with pytest.raises(ValueError):
                    layer(**kw)


@pytest.mark.gpu
def test_norm_without_gradients_stores_nothing(monkeypatch):
    asked = []
    real = ops.group_norm
    monkeypatch.setattr(ops, "group_norm", lambda *a, **kw: (asked.append(kw["save"]), real(*a, **kw))[1])
    x = torch.randn(2, 9, 32, device=DEV, requires_grad=True)
    with torch.no_grad():
        y = group_norm(x, 4)
    assert torch.equal(y, group_norm(x, 4).detach()) and asked == [None, "int8"]


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["linear", "norm"])
def test_checkpoints_go_with_the_backward_pass(what):
    """Once the backward pass is over its checkpoints are free, also while the loss is held, and a second pass is refused."""
    x = torch.randn(4, 1024, 512, device=DEV).bfloat16()
    w = torch.randn(512, 512, device=DEV).bfloat16().requires_grad_() if what == "linear" else torch.ones(512, device=DEV, requires_grad=True)
    w.grad = torch.zeros_like(w)
    layer = (lambda: linear(x, w)) if what == "linear" else (lambda: group_norm(x, 8, w))
    layer().sum().backward()                                     # the workspaces that torch's library calls keep for good
    before = torch.cuda.memory_allocated()
    loss = layer().sum()
    held = 4 * 1024 * (512 + 512 // 64)
    assert torch.cuda.memory_allocated() >= before + held
    loss.backward()
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() < before + held
    with pytest.raises(RuntimeError):
        loss.backward()


@pytest.mark.gpu
def test_linear_of_uneven_rows_and_of_nothing():
    """Inputs and gradients whose rows are not evenly spaced, gradients that are one expanded value, and no rows at all.  Two bf16
    roundings of sums in another order: 2 * 2^-8 of the value; fp32 sums of 48 terms below 16: 48 * 48 * 16 * 2^-24 = 2.2e-3 at the
    very most, of which signs leave far less: 1e-3."""
    near = dict(rtol=2 ** -7, atol=1e-3)
    x, w, b = _layer(torch.bfloat16, 60, 48, 40)
    base = x.detach().view(3, 20, 48)
    for x3 in (base.transpose(0, 1), base[:, :1].expand(3, 20, 48), base[:, ::2], base[:, :0], base[0, 0]):
        x3 = x3.detach().requires_grad_()
        for bias in (b, None):
            y = linear(x3, w, bias)
            assert torch.allclose(y, torch.nn.functional.linear(x3.detach().contiguous().view(-1, 48), w, bias).view(y.shape), **near)
            dy = torch.ones(1, dtype=y.dtype, device=DEV).expand(y.shape)
            dx, dw = torch.autograd.grad(y, (x3, w), dy)
            assert torch.allclose(dx, torch.mm(dy.reshape(-1, 40), w.detach()).view(x3.shape), **near)
            assert torch.equal(dw, ops.byte_linear_grad(dy.contiguous(), ops.byte_store(x3.detach().contiguous()))[0])


@pytest.mark.gpu
@pytest.mark.parametrize("shape,packs", [((5000, 1), True), ((3000, 3), False), ((64, 32, 1, 1), True), ((1, 4096), True),
                                         ((1000, 2, 8), False), ((1000, 9), True), ((1000, 16), True)])
def test_hooks_hold_only_what_gets_smaller(shape, packs):
    """bf16, groups of 32: a row takes 16 bytes of codes and one of its exponent at least, which is more than 3 or 8 values take as
    they are and less than 9 (a last dimension of one element counts as none)."""
    held = ByteCheckpoints("int8", 32, min_numel=1)
    x = torch.randn(shape, device=DEV).bfloat16()
    h = held.pack(x)
    assert (h is not x) == packs
    if packs:
        assert h.ck.nbytes < 2 * x.numel() and held.unpack(h).shape == x.shape
        flat = [n for n in shape if n != 1]
        assert torch.equal(held.unpack(h).view(flat), ops.byte_load(ops.byte_store(x.view(flat), "int8", 32)))


def _layer(dtype, rows, cols, outs, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen).to(dtype).to(DEV)
    w = (torch.randn(outs, cols, generator=gen) / cols ** 0.5).to(dtype).to(DEV)
    b = torch.randn(outs, generator=gen).to(dtype).to(DEV)
    return [t.requires_grad_() for t in (x, w, b)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("fmt,group", [("int8", 64), ("e4m3", 32)])
def test_linear_layer(dtype, fmt, group):
    """The output is the plain layer's, dx too; dW and db are what byte_linear_grad says, for inputs of more dimensions and
    for gradients that come as one expanded value."""
    x, w, b = _layer(dtype, 60, 48, 40)
    x3 = x.detach().view(3, 20, 48).requires_grad_()
    y = linear(x3, w, b, fmt, group)
    assert torch.equal(y, torch.nn.functional.linear(x3, w, b))
    dy = torch.randn(y.shape, generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
    dx, dw, db = torch.autograd.grad(y, (x3, w, b), dy)
    want_w, want_b = ops.byte_linear_grad(dy, ops.byte_store(x3.detach(), fmt, group), bias=True)
    assert torch.equal(dw, want_w) and torch.equal(db, want_b)
    assert torch.equal(dx, torch.matmul(dy, w.detach()))
    dw, db = torch.autograd.grad(linear(x3, w, b, fmt, group).sum(), (w, b))
    want_w, want_b = ops.byte_linear_grad(torch.ones_like(dy), ops.byte_store(x3.detach(), fmt, group), bias=True)
    assert torch.equal(dw, want_w) and torch.equal(db, want_b)
    # what needs no gradient is not computed or held
    y = linear(x3, w.detach(), None, fmt, group)
    assert torch.autograd.grad(y.sum(), x3)[0].shape == x3.shape
    y = linear(x3.detach(), w.detach(), b, fmt, group)
    assert torch.allclose(torch.autograd.grad(y.sum(), b)[0].float(), torch.full((40,), 60.0, device=DEV))


@pytest.mark.gpu
def test_linear_under_autocast():
    """fp32 parameters, a bf16 product: the weight's gradient comes back in fp32 from bf16 gradients."""
    x, w, b = _layer(torch.float32, 64, 48, 40)
    with torch.autocast(DEV, dtype=torch.bfloat16):
        y = linear(x, w, b)
    assert y.dtype == torch.bfloat16
    y.float().square().sum().backward()
    assert x.grad.dtype == w.grad.dtype == b.grad.dtype == torch.float32
    dy = (2 * y.detach().float()).bfloat16()
    want_w, want_b = ops.byte_linear_grad(dy, ops.byte_store(x.detach()), bias=True, dtype=torch.float32)
    assert torch.equal(w.grad, want_w) and torch.equal(b.grad, want_b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", [None, "int8", "e4m3"])
def test_group_norm_layer(dtype, fmt):
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(4, 6, 7, 40, generator=gen).to(dtype).to(DEV).requires_grad_()
    w, b = (torch.randn(40, generator=gen).to(dtype).to(DEV).requires_grad_() for _ in range(2))
    y = group_norm(x, 8, w, b, act="silu", fmt=fmt, group=32)
    dy = torch.randn(y.shape, generator=gen).to(dtype).to(DEV)
    got = torch.autograd.grad(y, (x, w, b), dy)
    y2, stats, ck = ops.group_norm(x.detach(), 8, w.detach().float(), b.detach().float(), act="silu", save=fmt, group=32)
    want = ops.group_norm_grad(dy, x.detach() if ck is None else ck, stats, 8, w.detach().float(), b.detach().float(), "silu")
    assert torch.equal(y, y2)
    for g, v, p in zip(got, want, (x, w, b)):
        assert g.dtype == p.dtype and g.shape == p.shape and torch.equal(g, v.to(p.dtype))
    (dx,) = torch.autograd.grad(group_norm(x, 8, w.detach(), None, fmt=fmt), x, dy)
    assert dx.shape == x.shape


def _block(x, p, fmt):
    """Group norm + SiLU, a pointwise convolution (a linear layer over the channels), a residual sum."""
    h = group_norm(x, 8, p[0], p[1], act="silu", fmt=fmt, group=32)
    h = linear(h, p[2], p[3], fmt, 32)
    h = group_norm(h, 4, p[4], p[5], act="relu", fmt=fmt, group=64)
    return x + linear(h, p[6], p[7], fmt, 64)


def _block_parameters(dtype):
    gen = torch.Generator().manual_seed(5)
    shapes = [(64,), (64,), (96, 64), (96,), (96,), (96,), (64, 96), (64,)]
    return [(torch.randn(s, generator=gen) * (0.1 if len(s) == 2 else 0.5) + (1.0 if i in (0, 4) else 0.0)).to(dtype).to(DEV).requires_grad_()
            for i, s in enumerate(shapes)]


def _block_in_64_bits(x, p, fmt, dy):
    """The block and its gradients from the formulas, with the inputs of the layers held as the codes stand for; every
    rounding but that of the codes left out."""
    def held(v, group):
        rows = v.detach().float().reshape(-1, v.shape[-1]).double().numpy()
        return torch.from_numpy(ref.decode(*ref.encode(rows, fmt, group), fmt, group)).view(v.shape)
    w = [t.detach().double().cpu() for t in p]
    x = x.detach().double().cpu()
    h1, m1, r1, _ = ref.norm(x, 8, w[0], w[1], 1e-5, "silu")
    h2 = h1 @ w[2].t() + w[3]
    h3, m3, r3, _ = ref.norm(h2, 4, w[4], w[5], 1e-5, "relu")
    y = x + h3 @ w[6].t() + w[7]
    flat = lambda v: v.reshape(-1, v.shape[-1])  # noqa: E731
    dw6, db7, d3 = flat(dy).t() @ flat(held(h3, 64)), flat(dy).sum(0), dy @ w[6]
    d2, dw4, db5, _, _ = ref.norm_grad(d3, held(h2, 64), m3, r3, w[4], w[5], "relu")
    dw2, db3, d1 = flat(d2).t() @ flat(held(h1, 32)), flat(d2).sum(0), d2 @ w[2]
    dx, dw0, db1, _, _ = ref.norm_grad(d1, held(x, 32), m1, r1, w[0], w[1], "silu")
    return y, [dy + dx, dw0, db1, dw2, db3, dw4, db5, dw6, db7]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_a_block_against_the_formulas(fmt):
    """All operators in a row in fp32.  The codes of the inner layers' inputs are rounded from values that differ in
    their last bits from the reference's: a code next to a tie moves by one step then (at most 2^-6 of its group's largest
    value for int8, 2^-3 of itself for e4m3) in about one value of 10^4, and a ReLU next to its border changes sides.  Both are
    bounded in the 2-norm by the square root of their share: 1e-2 of a step of 1/8, 2e-3 with a margin of two."""
    p = _block_parameters(torch.float32)
    gen = torch.Generator().manual_seed(6)
    x = torch.randn(2, 49, 64, generator=gen).to(DEV).requires_grad_()
    dy = torch.randn(2, 49, 64, generator=gen)
    y = _block(x, p, fmt)
    got = torch.autograd.grad(y, [x, *p], dy.to(DEV))
    want_y, want = _block_in_64_bits(x, p, fmt, dy.double())
    assert float((y.detach().double().cpu() - want_y).norm() / want_y.norm()) < 1e-5
    for g, v in zip(got, want):
        assert float((g.double().cpu() - v).norm() / v.norm()) < 2e-3


@pytest.mark.gpu
def test_gradients_are_near_the_uncompressed_ones():
    """int8 holds a value to 1/127 of its group's largest: the smooth part of the gradients differs by a few times that in the
    2-norm.  The ReLU adds its border: the largest of 64 normal values is about 3 deviations, a step at most 3 / 64 of
    one and the mean error a quarter of that, 0.012; with the normal density 0.4 at the border a share of 0.005 of the
    values changes sides, 0.01 of those that pass, which is 0.1 in the 2-norm."""
    p = _block_parameters(torch.float32)
    gen = torch.Generator().manual_seed(7)
    x = torch.randn(4, 100, 64, generator=gen).to(DEV).requires_grad_()
    dy = torch.randn(4, 100, 64, generator=gen).to(DEV)
    got = torch.autograd.grad(_block(x, p, "int8"), [x, *p], dy)
    h = x
    for k, (g, act) in enumerate(((8, torch.nn.functional.silu), (4, torch.relu))):
        h = act(torch.nn.functional.group_norm(h.transpose(1, 2), g, p[4 * k], p[4 * k + 1]).transpose(1, 2))
        h = torch.nn.functional.linear(h, p[4 * k + 2], p[4 * k + 3])
    want = torch.autograd.grad(x + h, [x, *p], dy)
    for a, b in zip(got, want):
        assert float((a - b).norm() / b.norm()) < 5 / 127 + 0.1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_hooks(dtype):
    """A convolution in channels_last and a linear layer under the hooks: the backward pass receives what the checkpoints
    stand for, as often as it is walked."""
    torch.manual_seed(11)
    conv = torch.nn.Conv2d(16, 24, 3, padding=1).to(DEV, dtype, memory_format=torch.channels_last)
    head = torch.nn.Linear(24, 10).to(DEV, dtype)
    x = torch.randn(4, 16, 20, 20, device=DEV).to(dtype).to(memory_format=torch.channels_last).requires_grad_()
    held = ByteCheckpoints("int8", 32, min_numel=1 << 10)
    held.skip_parameters([*conv.parameters(), *head.parameters()])
    with held.hooks():
        mid = conv(x)
        loss = head(mid.permute(0, 2, 3, 1)).float().square().sum()
    assert held.stats["packed"] >= 2 and held.stats["held_bytes"] < 0.6 * held.stats["raw_bytes"]
    first = torch.autograd.grad(loss, [x, *conv.parameters(), *head.parameters()], retain_graph=True)
    again = torch.autograd.grad(loss, [x, *conv.parameters(), *head.parameters()])
    x2 = ops.byte_load(ops.byte_store(x.detach().permute(0, 2, 3, 1), "int8", 32)).permute(0, 3, 1, 2)
    plain = torch.autograd.grad(head(conv(x).permute(0, 2, 3, 1)).float().square().sum(), [x, *conv.parameters(), *head.parameters()])
    for a, b, c in zip(first, again, plain):
        assert torch.allclose(a.float(), b.float(), rtol=1e-2, atol=1e-3 * float(b.float().abs().max()))
        assert float((a.float() - c.float()).norm()) <= 0.05 * float(c.float().norm())
    h = held.pack(x.detach())
    assert torch.equal(held.unpack(h), x2) and held.unpack(h).stride() == x.stride()
    assert isinstance(held.pack(x.detach()[:, :, ::2]), torch.Tensor) and held.pack(conv.weight) is conv.weight


@pytest.mark.gpu
def test_replays_from_a_graph():
    """Store, load, both gradients and both directions of the norm captured once; every replay on changed inputs, with eager
    calls between them, gives the eager results."""
    gen = torch.Generator().manual_seed(13)
    sets = [[torch.randn(s, generator=gen).bfloat16().to(DEV) for s in ((3, 2000, 96), (3, 2000, 96), (6000, 40))] for _ in range(3)]
    w, b = (torch.randn(96, generator=gen).to(DEV) for _ in range(2))

    def step(x, dy, dz):
        y, stats, ck = ops.group_norm(x, 8, w, b, act="silu", save="int8", group=32)
        dx, dw, db = ops.group_norm_grad(dy, ck, stats, 8, w, b, "silu")
        held = ops.byte_store(y, "e4m3", 32)
        gw, gb = ops.byte_linear_grad(dz, held, bias=True)
        return y, stats, ck.buf, dx, dw, db, held.buf, ops.byte_load(held), gw, gb

    want = [[t.clone() for t in step(*s)] for s in sets]
    ins = [torch.empty_like(t) for t in sets[0]]
    side = torch.cuda.Stream()
    for a, v in zip(ins, sets[0]):
        a.copy_(v)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*ins)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):                                            # two graphs of the same calls: each has its own workspaces
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(step(*ins))
        graphs.append(g)
    for v in (1, 2, 0, 1):
        for a, s in zip(ins, sets[v]):
            a.copy_(s)
        for o in outs:
            for t in o:
                t.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o in outs:
            for t, u in zip(o, want[v]):
                assert torch.equal(t, u)
        step(*sets[(v + 1) % 3])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("frozen", [False, True])
def test_layers_replay_from_a_graph(dtype, frozen):
    """A block of the layers, forward and backward through autograd, captured once; every replay on changed inputs, with
    eager calls of the same block between, gives the eager results.  frozen: only the biases of the linear layers learn."""
    p = _block_parameters(dtype)
    learn = [p[3], p[7]] if frozen else p
    if frozen:
        for k in (0, 1, 2, 4, 5, 6):
            p[k].requires_grad_(False)
    gen = torch.Generator().manual_seed(19)
    sets = [[torch.randn(6, 1000, 64, generator=gen).to(dtype).to(DEV) for _ in range(2)] for _ in range(3)]

    def step(x, dy):
        x = x.detach().requires_grad_()
        y = _block(x, p, "int8")
        return [y.detach(), *torch.autograd.grad(y, [x, *learn], dy)]

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


@pytest.mark.gpu
def test_two_streams_at_once():
    """The same calls on two streams, their buffers apart: the results of each alone."""
    gen = torch.Generator().manual_seed(17)
    sets = [(torch.randn(4, 3000, 64, generator=gen).to(DEV), torch.randn(12000, 80, generator=gen).to(DEV)) for _ in range(2)]

    def step(x, dz):
        y, stats, ck = ops.group_norm(x, 8, act="silu", save="int8")
        return [*ops.group_norm_grad(x, ck, stats, 8, act="silu"), *ops.byte_linear_grad(dz, ck, bias=True), y]

    want = [[t.clone() for t in step(*s)] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = []
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(step(*s))
        torch.cuda.synchronize()
        for g, v in zip(got, want):
            for t, u in zip(g, v):
                assert torch.equal(t, u)
