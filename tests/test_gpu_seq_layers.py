"""Layers that keep their input in 8 bits, the recurrent layer and block, and a stack of them as a network would use it."""
import copy

import numpy as np
import pytest
import torch

from paper_2504_06881_b200 import inputs, layers as tlayers, nn as tnn, tconv, tconv3d

pytestmark = pytest.mark.gpu


def _layer(kind, mode, dtype, checkpoint, seed=0):
    torch.manual_seed(seed)
    args = dict(mode=mode, dtype=dtype, checkpoint=checkpoint)
    made = {"dense": lambda: tnn.TropicalConv2d(5, 7, 3, padding=1, **args),
            "wide": lambda: tnn.TropicalConv2d(4, 6, 5, stride=2, padding=2, **args),
            "depthwise": lambda: tnn.TropicalDepthwiseConv2d(6, 3, padding=1, **args),
            "signal": lambda: tnn.TropicalConv1d(4, 8, 3, padding=1, **args),
            "long": lambda: tnn.TropicalConv1d(2, 8, 21, stride=2, padding=10, **args),
            "volume": lambda: tnn.TropicalConv3d(3, 4, 3, padding=1, **args)}[kind]().cuda()
    shape = {"dense": (3, 5, 9, 11), "wide": (2, 4, 16, 16), "depthwise": (2, 6, 14, 14), "signal": (3, 4, 77), "long": (2, 2, 300),
             "volume": (2, 3, 6, 7, 8)}[kind]
    with torch.no_grad():
        for p in made.parameters():
            p.uniform_(-0.5, 0.5)
    return made, torch.randn(shape, device="cuda")


def _run(layer, x, **kw):
    x = x.detach().requires_grad_(True)
    y = layer(x, **kw)
    torch.manual_seed(9)
    g = torch.randn_like(y)
    names = ["x"] + [n for n, _ in layer.named_parameters()]
    return y.detach(), dict(zip(names, torch.autograd.grad(y, [x] + list(layer.parameters()), g))), g


@pytest.mark.parametrize("kind", ["dense", "wide", "depthwise", "signal", "long", "volume"])
@pytest.mark.parametrize("mode", ["max_plus", "compound", "parallel"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layers_with_kept_inputs(kind, mode, dtype):
    """The forward and all gradients but those of alpha and beta bit for bit; those differ from the full ones by no more than
    the input's rounding carries over: half a unit of its block, times the upstream gradient, summed."""
    plain, x = _layer(kind, mode, dtype, None)
    kept, _ = _layer(kind, mode, dtype, "q8")
    kept.load_state_dict(plain.state_dict())
    y0, g0, up = _run(plain, x)
    y1, g1, _ = _run(kept, x)
    assert torch.equal(y0, y1)
    for n in g0:
        if n.rsplit(".", 1)[-1] not in ("alpha", "beta"):
            assert torch.equal(g0[n], g1[n]), n
        else:
            # (every |x| < 6: units of 2^-4 at most, so that a branch value is off by 2^-5 at most; bf16 taps add a rounding
            # of values below 7, 2^-6, on either side; and the sums' own rounding, twice 1e-5 of their terms below 7)
            off = 2.0 ** -5 + (2 * 2.0 ** -6 if dtype == "bf16" else 0) + 2 * 7e-5
            assert x.abs().max() < 6
            per_out = up.abs().sum([d for d in range(up.dim()) if d != 1])
            bound = off * (per_out if g0[n].dim() == 1 else per_out[:, None])
            assert ((g0[n] - g1[n]).abs() <= bound * (1 + 2.0 ** -7)).all(), n
    # the input's 8-bit form made elsewhere
    y2, g2, _ = _run(kept, x, stored=tnn.q8_store(x if dtype == "f32" else x.bfloat16()))
    assert torch.equal(y2, y0) and all(torch.equal(g1[n], g2[n]) for n in g1)
    with torch.no_grad():
        assert torch.equal(kept(x), y0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["compound", "parallel"])
def test_kept_gradients_are_those_over_the_restored_input(mode, dtype):
    """grad_alpha and grad_beta against the library's backward with the restored input and the true winners."""
    dt = tconv.TORCH_DTYPE[dtype]
    layer, x = _layer("dense", mode, dtype, "q8")
    _, grads, up = _run(layer, x)
    d = inputs.layer(*x.shape, 7, 3, 3, pad=1, mode=mode, dtype=dtype)
    w, w2 = layer.weight.detach().to(dt), None if layer.weight2 is None else layer.weight2.detach().to(dt)
    a, b = layer.alpha.detach(), layer.beta.detach()
    xc = x.to(dt)
    _, winners = tconv.forward(d, xc, w, w2, a, b, layer.bias.detach(), want_winners=True)
    want = tconv.backward(d, tnn.q8_store(xc).restore(), w, up.to(dt), w2, a, b, winners)
    assert torch.equal(grads["alpha"], want["grad_alpha"]) and torch.equal(grads["beta"], want["grad_beta"])
    layer, x = _layer("volume", mode, dtype, "q8")
    _, grads, up = _run(layer, x)
    d = inputs.layer3d(*x.shape, 4, pad=1, mode=mode, dtype=dtype)
    w, w2 = layer.weight.detach().to(dt), None if layer.weight2 is None else layer.weight2.detach().to(dt)
    a, b = layer.alpha.detach(), layer.beta.detach()
    xc = x.to(dt)
    _, winners = tconv3d.forward(d, xc, w, w2, a, b, layer.bias.detach(), want_winners=True)
    want = tconv3d.backward(d, tnn.q8_store(xc).restore(), w, up.to(dt), w2, a, b, winners)
    assert torch.equal(grads["alpha"], want["grad_alpha"]) and torch.equal(grads["beta"], want["grad_beta"])


def _saved_bytes(fn):
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t.nbytes), t)[1], lambda t: t):
        out = fn()
    return sum(seen), out


def test_what_is_kept_is_smaller_and_survives_hooks():
    layer, _ = _layer("depthwise", "compound", "f32", None)
    kept, _ = _layer("depthwise", "compound", "f32", "q8")
    x = torch.randn(8, 6, 56, 56, device="cuda", requires_grad=True)
    full, _ = _saved_bytes(lambda: layer(x))
    small, _ = _saved_bytes(lambda: kept(x))
    assert full - small >= x.nbytes - x.numel() * 1.05
    s = torch.randn(2, 8, 4096, device="cuda", requires_grad=True)
    f, _ = _saved_bytes(lambda: tnn.gated_scan(s, s))
    q, _ = _saved_bytes(lambda: tnn.gated_scan(s, s, checkpoint="q8"))
    assert f >= 2 * s.nbytes and q <= 2.2 * s.numel()
    w = torch.ones(8, device="cuda")
    f, _ = _saved_bytes(lambda: tnn.rms_norm(s, w).y)
    q, _ = _saved_bytes(lambda: tnn.rms_norm(s, w, checkpoint="q8").y)
    assert f >= s.nbytes and q <= 1.7 * s.numel()
    for fn in (lambda: kept(x), lambda: tnn.gated_scan(x[:, :, 0], x[:, :, 1], checkpoint="q8")[0], lambda: tnn.gated_scan(x[:, :, 0])[0],
               lambda: tnn.rms_norm(x, torch.ones(6, device="cuda"), x, checkpoint="q8").y, lambda: tnn.rms_norm(x, torch.ones(6, device="cuda"), x).y):
        want = torch.autograd.grad(fn().square().sum(), x)[0]
        with torch.autograd.graph.save_on_cpu():
            y = fn()
        assert torch.equal(torch.autograd.grad(y.square().sum(), x)[0], want)
        got = torch.utils.checkpoint.checkpoint(lambda _: fn(), x, use_reentrant=False)
        assert torch.equal(torch.autograd.grad(got.square().sum(), x)[0], want)


def test_layer_refusals():
    layer, x = _layer("dense", "compound", "f32", None)
    kept, _ = _layer("dense", "compound", "f32", "q8")
    with pytest.raises(ValueError, match="checkpoint='q8'"):
        layer(x, stored=tnn.q8_store(x))
    with pytest.raises(ValueError, match="codes"):
        kept(x.requires_grad_(True), stored=tnn.q8_store(x[:2].contiguous()))
    with pytest.raises(ValueError, match="checkpoint must be"):
        tnn.TropicalConv1d(2, 2, 3, checkpoint="q4")
    with pytest.raises(NotImplementedError, match="traced"):
        torch.jit.trace(kept, x.detach(), check_trace=False)
    tnn.TropicalConvFn.events = []
    try:
        with pytest.raises(ValueError, match="events"):
            kept(x)
    finally:
        tnn.TropicalConvFn.events = None
    old = copy.deepcopy(layer)
    del old.__dict__["checkpoint"]                    # a layer pickled before it could keep its input in 8 bits
    assert torch.equal(old(x), layer(x)) and "checkpoint" not in repr(old)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("k,stride,L", [(3, 1, 61), (21, 2, 300), (3, 1, 1)])
def test_recurrent_layer_is_its_parts(k, stride, L, checkpoint, dtype):
    torch.manual_seed(2)
    rec = tlayers.TropicalRecurrent1d(4, 6, k, stride, padding=k // 2, dtype=dtype, checkpoint=checkpoint).cuda()
    assert (rec.conv.conv.bias[6:] == 2).all() and (rec.conv.conv.bias[:6] == 0).all()
    x = torch.randn(3, 4, L, device="cuda", requires_grad=True)
    h0 = torch.randn(3, 6, device="cuda", requires_grad=True)
    y, last = rec(x, h0)
    both = rec.conv(x)
    y2, last2 = tnn.gated_scan(both[:, :6].contiguous(), both[:, 6:].contiguous(), h0, checkpoint=checkpoint)
    assert torch.equal(y, y2) and torch.equal(last, last2)
    ins = [x, h0] + list(rec.parameters())
    up = (torch.randn_like(y), torch.randn_like(last))
    for a, b in zip(torch.autograd.grad((y, last), ins, up), torch.autograd.grad((y2, last2), ins, up)):
        assert torch.equal(a, b)


def _conv64(x, conv):
    """The compound 3-tap layer with padding 1 in 64 bits."""
    c = conv.conv
    w, a, b = (t.double().squeeze() for t in (c.weight, c.alpha, c.beta))
    t = torch.nn.functional.pad(x, (1, 1)).unfold(2, 3, 1).unsqueeze(1) + w[None, :, :, None, :]
    return (a[None, :, :, None] * t.amin(-1) + b[None, :, :, None] * t.amax(-1)).sum(2) + c.bias.double()[None, :, None]


def _scan64(both, lengths):
    x, g = both.chunk(2, 1)
    f = torch.sigmoid(g)
    h, ys = torch.zeros_like(x[..., 0]), []
    for t in range(x.shape[2]):
        live = (t < lengths)[:, None]
        h = torch.where(live, f[..., t] * h + (1 - f[..., t]) * x[..., t], h)
        ys.append(torch.where(live, h, torch.zeros_like(h)))
    return torch.stack(ys, -1)


def _norm64(s, norm):
    return s / torch.sqrt((s * s).mean(1, keepdim=True) + norm.eps) * norm.weight.double()[None, :, None]


def _network(C, depth, checkpoint, dtype="f32"):
    torch.manual_seed(4)
    net = torch.nn.ModuleList([tlayers.TropicalRecurrentBlock1d(C, dtype=dtype, checkpoint=checkpoint) for _ in range(depth)] +
                              [tlayers.RMSNorm(C, checkpoint=checkpoint)]).cuda()
    with torch.no_grad():
        for n, p in net.named_parameters():
            if n.endswith(("alpha", "beta")):
                p.mul_(torch.empty_like(p).uniform_(0.5, 1.5))
            elif n.endswith("norm.weight"):
                p.uniform_(0.7, 1.3)
    return net


def _forward(net, x, lengths):
    stream = None
    for block in net[:-1]:
        x, stream = block(x, stream, lengths)
    return net[-1](x, stream)[0]


def test_stack_against_64_bits():
    """Three blocks and a last norm on a ragged batch, forward and every gradient, in fp32.  Each operation is off by some 1e-6 of
    its values' size at most (sums of 16 channels, gates to 2e-6); none stretches a difference by more than ten (norms of
    a stream of size one, convolutions whose alpha and beta sum to one, recurrences that average), and there are ten in a row,
    most of them added to the stream rather than passed on: 1e-4 of the result's norm.  A tap that wins by less than that in 64
    bits may lose in 32, which moves a gradient by its whole term: the taps of 3 * 16 * 40 * 32 * 2 choices that lie within 1e-6
    of each other are 1e-6 of them, less than one."""
    net = _network(16, 3, None)
    x = torch.randn(3, 16, 40, device="cuda", requires_grad=True)
    lengths = torch.tensor([40, 17, 0], dtype=torch.int32, device="cuda")
    y = _forward(net, x, lengths)
    up = torch.randn_like(y)
    ins = [x] + list(net.parameters())
    got = torch.autograd.grad(y, ins, up)
    x64, branch, stream = x.double(), None, None
    for block in net[:-1]:
        stream = x64 if branch is None else stream + branch
        branch = _scan64(_conv64(_norm64(stream, block.norm), block.rec.conv), lengths)
    y64 = _norm64(stream + branch, net[-1])
    want = torch.autograd.grad(y64, ins, up.double())
    for a, b in zip((y,) + got, (y64,) + want):
        assert (a.double() - b).norm() <= 1e-4 * b.norm() + 1e-9


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_stack_with_kept_activations(dtype):
    """The same network with its activations in 8 bits: the forward bit for bit, finite gradients of every parameter, and a
    training step in a captured graph gives the eager one's weights."""
    x = torch.randn(2, 16, 333, device="cuda")
    lengths = torch.tensor([333, 200], dtype=torch.int32, device="cuda")
    nets = [_network(16, 2, ck, dtype) for ck in (None, "q8")]
    outs = [_forward(n, x, lengths) for n in nets]
    assert torch.equal(*outs)
    up = torch.randn_like(outs[0])
    grads = [torch.autograd.grad(y, list(n.parameters()), up) for y, n in zip(outs, nets)]
    for a, b in zip(*grads):
        assert torch.isfinite(b).all() and a.shape == b.shape
    with torch.no_grad():
        assert torch.equal(_forward(nets[1], x, lengths), outs[0])

    def step(net):
        loss = (_forward(net, x, lengths) * up).sum()
        with torch.no_grad():
            for p, g in zip(net.parameters(), torch.autograd.grad(loss, list(net.parameters()))):
                p.add_(g, alpha=-1e-3)

    eager, captured = _network(16, 2, "q8", dtype), _network(16, 2, "q8", dtype)
    for _ in range(3):
        step(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(captured)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager.parameters(), captured.parameters()))
