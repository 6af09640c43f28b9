"""Layers with checkpoint="q8": what they keep where no gradient of alpha or beta is wanted, and what the recurrent block's
convolution is handed."""
import pytest
import torch

from paper_2504_06881_b200 import inputs, layers as tlayers, nn as tnn, tconv, tconv3d

pytestmark = pytest.mark.gpu

SHAPES = {"dense": (3, 5, 9, 11), "wide": (2, 4, 16, 16), "depthwise": (2, 6, 14, 14), "windows": (2, 6, 13, 15), "signal": (3, 4, 77),
          "long": (2, 2, 300), "volume": (2, 3, 6, 7, 8)}


def _layer(kind, checkpoint, **args):
    torch.manual_seed(0)
    args = dict(args, checkpoint=checkpoint)
    made = {"dense": lambda: tnn.TropicalConv2d(5, 7, 3, padding=1, **args),
            "wide": lambda: tnn.TropicalConv2d(4, 6, 5, stride=2, padding=2, **args),
            "depthwise": lambda: tnn.TropicalDepthwiseConv2d(6, 3, padding=1, **args),
            "windows": lambda: tnn.TropicalDepthwiseConv2d(6, (2, 3), stride=2, **args),
            "signal": lambda: tnn.TropicalConv1d(4, 8, 3, padding=1, **args),
            "long": lambda: tnn.TropicalConv1d(2, 8, 21, stride=2, padding=10, **args),
            "volume": lambda: tnn.TropicalConv3d(3, 4, 3, padding=1, **args)}[kind]().cuda()
    with torch.no_grad():
        for p in made.parameters():
            p.uniform_(-0.5, 0.5)
    return made


def _kept(fn):
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t.nbytes), t)[1], lambda t: t):
        out = fn()
    return sum(seen), out


def _launches():
    return tconv.tconv_launch_count() + tconv3d.tconv3d_launch_count()


# what leaves no gradient of alpha or beta to be wanted
NONE_WANTED = {"max_plus": dict(mode="max_plus"), "min_plus": dict(mode="min_plus"), "0p": dict(mode="compound", params="0p"),
               "fixed": dict(mode="parallel", params="fixed", fixed=(1.0, -1.0)), "frozen": dict(mode="compound")}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", NONE_WANTED)
@pytest.mark.parametrize("kind", SHAPES)
def test_nothing_is_kept_for_gradients_that_are_not_wanted(kind, how, dtype):
    plain, lean = (_layer(kind, ck, dtype=dtype, **NONE_WANTED[how]) for ck in (None, "q8"))
    x = torch.randn(SHAPES[kind], device="cuda")
    for m in (plain, lean):
        if how == "frozen":
            for n, p in m.named_parameters():
                p.requires_grad_(n.rsplit(".", 1)[-1] not in ("alpha", "beta"))
    results = []
    for m in (plain, lean):
        for wanted in (True, False):                      # of x itself (a first layer's is not)
            xi = x.clone().requires_grad_(wanted)
            before = _launches()
            nbytes, y = _kept(lambda: m(xi))
            params = [p for p in m.parameters() if p.requires_grad]
            torch.manual_seed(1)
            grads = torch.autograd.grad(y, [xi] * wanted + params, torch.randn_like(y))
            results.append((y, grads, nbytes, _launches() - before))
    for (y, grads, full, most), (y2, grads2, kept, launches) in zip(results[:2], results[2:]):
        assert torch.equal(y, y2) and len(grads) == len(grads2)
        assert all(torch.equal(a, b) for a, b in zip(grads, grads2))
        xbytes = x.numel() * (4 if dtype == "f32" else 2)
        assert kept == full - xbytes and launches <= most
    # anomaly mode looks at every gradient the node returns, the unwanted ones too
    with torch.autograd.detect_anomaly(check_nan=True):
        xi = x.clone().requires_grad_(True)
        y = lean(xi, stored=tnn.q8_store(x))
        torch.manual_seed(1)
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, [xi] + params, torch.randn_like(y)), results[0][1]))
    with torch.autograd.graph.save_on_cpu():
        y = lean(xi)
    torch.manual_seed(1)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, [xi] + params, torch.randn_like(y)), results[0][1]))
    with pytest.raises(ValueError, match="codes"):
        lean(xi, stored=tnn.q8_store(torch.cat([x, x])))


@pytest.mark.parametrize("kind", ["dense", "depthwise", "volume"])
@pytest.mark.parametrize("half", ["alpha", "beta"])
def test_one_of_alpha_and_beta_wanted(kind, half):
    """One of the two is enough for the input to be kept, and its gradient is the one of a layer that learns both."""
    layer = _layer(kind, "q8", mode="parallel")
    x = torch.randn(SHAPES[kind], device="cuda", requires_grad=True)
    up = torch.randn_like(layer(x))
    names = [n for n, _ in layer.named_parameters()]
    both = dict(zip(names, torch.autograd.grad(layer(x), list(layer.parameters()), up)))
    for n, p in layer.named_parameters():
        p.requires_grad_(n.rsplit(".", 1)[-1] != ("alpha" if half == "beta" else "beta"))
    got = dict(layer.named_parameters())
    got = {n: p for n, p in got.items() if p.requires_grad}
    for n, g in zip(got, torch.autograd.grad(layer(x), list(got.values()), up)):
        assert torch.equal(g, both[n]), n


def test_backward_holds_no_copy_of_an_input_it_does_not_read():
    """A max-plus layer's backward allocates the input's gradient and no second tensor of its size."""
    layer = _layer("wide", "q8", mode="max_plus")
    x = torch.randn(64, 4, 128, 128, device="cuda", requires_grad=True)
    peaks = []
    for m in (_layer("wide", None, mode="max_plus"), layer):
        y = m(x)
        up = torch.randn_like(y)
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        held = torch.cuda.memory_allocated()
        g = torch.autograd.grad(y, [x] + list(m.parameters()), up)
        torch.cuda.synchronize()
        peaks.append(torch.cuda.max_memory_allocated() - held)
        del y, up, g
    assert peaks[1] <= peaks[0] + 4096


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("first", [True, False])
def test_block_with_kept_activations(first, dtype):
    """The recurrent block with checkpoint="q8" is its parts, the convolution's input kept as the norm's own 8-bit output (of y in
    fp32, before the convolution's rounding): every gradient bit for bit, those of alpha and beta over that form's values.

    Against the block that keeps everything: a restored value is off by 1/127 of its block's largest at most, some 0.05 for normalised
    signals whose largest is 6.  f (1 - f) moves by as much relatively, f's products over the 1 / (1 - f) positions that a state
    lasts by as much again, h - x and a branch value by 0.05 each; with the norm's stream, a quarter of a gradient's norm at most."""
    torch.manual_seed(5)
    blocks = [tlayers.TropicalRecurrentBlock1d(16, dtype=dtype, checkpoint=ck).cuda() for ck in ("q8", None)]
    with torch.no_grad():
        for n, p in blocks[0].named_parameters():
            p.mul_(torch.empty_like(p).uniform_(0.5, 1.5))
    blocks[1].load_state_dict(blocks[0].state_dict())
    block = blocks[0]
    x = torch.randn(2, 16, 333, device="cuda", requires_grad=True)
    r = None if first else torch.randn(2, 16, 333, device="cuda", requires_grad=True)
    lengths = torch.tensor([333, 200], dtype=torch.int32, device="cuda")
    ups = [torch.randn_like(x)] + [torch.randn_like(x)] * (not first)

    def grads(of, block):
        y, stream = of(block)
        ins = [x] + [r] * (not first) + list(block.parameters())
        return (y, stream) + torch.autograd.grad([y] + [stream] * (not first), ins, ups)

    inner = block.rec.conv.conv                           # the 1 x 3 windows of the signal's layer
    seen = {}

    def by_hand(b):
        n = tnn.rms_norm(x, b.norm.weight, r, b.norm.eps, "both", "q8")
        both = inner(n.y.unsqueeze(2), n.q8).squeeze(2)
        both.register_hook(lambda g: seen.update(grad=g.detach().clone()))
        seen.update(n=n)
        return tnn.gated_scan(both, None, None, lengths, "q8")[0], n.stream

    got = grads(lambda b: b(x, r, lengths), block)
    hand = grads(by_hand, block)
    assert len(got) == len(hand) and all(torch.equal(a, b) for a, b in zip(got, hand))
    dt = tconv.TORCH_DTYPE[dtype]
    d = inputs.layer(2, 16, 1, 333, 32, 1, 3, pad=(0, 1), mode="compound", dtype=dtype)
    xc, w = seen["n"].y.detach().to(dt).unsqueeze(2), inner.weight.detach().to(dt)
    a, b = inner.alpha.detach(), inner.beta.detach()
    _, winners = tconv.forward(d, xc, w, None, a, b, inner.bias.detach(), want_winners=True)
    want = tconv.backward(d, seen["n"].q8.restore(dt).unsqueeze(2), w, seen["grad"].to(dt).unsqueeze(2), None, a, b, winners)
    named = dict(zip([n for n, _ in block.named_parameters()], got[-len(list(block.parameters())):]))
    assert torch.equal(named["rec.conv.conv.alpha"], want["grad_alpha"]) and torch.equal(named["rec.conv.conv.beta"], want["grad_beta"])
    full = grads(lambda b: b(x, r, lengths), blocks[1])
    assert torch.equal(got[0], full[0]) and torch.equal(got[1], full[1])
    for k, (u, v) in enumerate(zip(got[2:], full[2:])):
        assert v.norm() > 0 and (u - v).norm() <= 0.25 * v.norm(), k
