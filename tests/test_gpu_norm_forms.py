"""Every form of the RMS norm's kernels against its plain 64-bit form, over enough positions that a block goes from tile to tile."""
import pytest
import torch

import norm_forms
import seq_ref as ref
from paper_2504_06881_b200 import nn as tnn, tconv
from test_gpu_seq import _q8_close

pytestmark = pytest.mark.gpu
DT = tconv.TORCH_DTYPE


def _np(t):
    return t.detach().double().cpu().numpy()


def _q8(t, rows, inner):
    """(values, units [rows, blocks]) of a finite tensor's 8-bit form, in 64 bits."""
    b = torch.nn.functional.pad(t.double().reshape(rows, inner), (0, -inner % 32)).reshape(rows, -1, 32)
    m, k = torch.frexp(b.abs().amax(-1))                  # amax = m 2^k, 1/2 <= m < 1
    e = torch.where(m == 0, torch.full_like(k, -126), k - 7 + (m >= 127.5 / 128).int()).clamp(-126, 121)
    unit = torch.ldexp(torch.ones_like(m), e)
    return (torch.round(b / unit[..., None]).clamp(-127, 127) * unit[..., None]).reshape(rows, -1)[:, :inner].reshape(t.shape), unit


def _near(got, want, off, what):
    assert ((got.detach().double() - want).abs() <= off + 1e-30).all(), what


def _weight_depth(N, P):
    """Roundings that a term of grad_weight goes through: its block's (warp's) tiles in turn, eight values of a tile at most, a
    shuffle of five; the 1184 partial sums at most by eights, and the eight.  148 blocks at least where there are as many tiles."""
    tiles = N * -(-P // 32) if P > 1 else -(-N // 4)
    return 8 * -(-tiles // 148) + 5 + 148 + 8 + 4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual,checkpoint", [(False, None), (True, None), (False, "q8"), (True, "q8")])
@pytest.mark.parametrize("N,C,P", norm_forms.MANY + norm_forms.FEW)
def test_forms(N, C, P, residual, checkpoint, dtype):
    gen = torch.Generator("cuda").manual_seed(N + C + P)
    shape, eps = (N, C) if P == 1 else (N, C, P), 1e-5
    make = lambda scale=1.0: (scale * torch.randn(shape, device="cuda", generator=gen)).to(DT[dtype])
    x, r, gy, gs = make().requires_grad_(True), make(2.0).requires_grad_(True) if residual else None, make(), make()
    w = (1 + 0.3 * torch.randn(C, device="cuda", generator=gen)).requires_grad_(True)
    ins, ups = [x, w] + [r] * residual, [gy] + [gs] * residual

    def run(x, r, ups):
        o = tnn.rms_norm(x, w, r, eps, output="both", checkpoint=checkpoint)
        return o, torch.autograd.grad([o.y] + [o.stream] * residual, [x, w] + [r] * residual, ups)

    o, grads = run(x, r, ups)
    stream = (x.float() + r.float()).to(DT[dtype]).detach() if residual else x.detach()
    assert torch.equal(o.stream, stream)
    assert not residual or torch.equal(grads[0], grads[2])
    # the definition in 64 bits, with the first-order bounds of seq_ref.norm
    EPS, half, rows, inner = ref.EPS, ref.HALF[dtype], *((N * C, P) if P > 1 else (N, C))
    s, g, wd = stream.double(), gy.double(), w.detach().double().view((1, C) + (1,) * (len(shape) - 2))
    rstd, er = 1 / torch.sqrt((s * s).mean(1, keepdim=True) + eps), (C + 8) * EPS
    y = s * rstd * wd
    ey = y.abs() * (er + 4 * EPS)
    _near(o.y, y, ey + half * (y.abs() + ey), "y")
    z = (_q8(s, rows, inner)[0] if checkpoint else s) * rstd
    m = (wd * g * z).mean(1, keepdim=True)
    em = (wd * g * z).abs().mean(1, keepdim=True) * ((C + 4) * EPS + er)
    d = rstd * (wd * g - z * m)
    ed = rstd * ((wd * g).abs() * (er + 4 * EPS) + (z * m).abs() * (2 * er + 6 * EPS) + z.abs() * em)
    if residual:
        d = d + gs.double()
        ed = ed + EPS * d.abs()
    _near(grads[0], d, ed + half * (d.abs() + ed), "grad_x")
    over = [k for k in range(len(shape)) if k != 1]
    _near(grads[1], (g * z).sum(over), (g * z).abs().sum(over) * ((_weight_depth(N, P) + 4) * EPS + er), "grad_weight")
    # the 8-bit form of a y known up to ey: the unit of some value within it, values within half a unit and it
    units = torch.ldexp(torch.ones(o.q8.scales.shape, device="cuda", dtype=torch.float64), o.q8.scales.int() - 127)
    lo, hi = (_q8(v, rows, inner)[1] for v in ((y.abs() - ey).clamp(min=0), y.abs() + ey))
    assert ((units >= lo) & (units <= hi)).all()
    wide = units.repeat_interleave(32, 1)[:, :inner].reshape(shape)
    _near(o.q8.restore(torch.float32), y, 0.5 * wide + ey, "q8")
    # a position's values are its own affair: the same, bit for bit, in a batch that gives each block one tile at most
    few = max(1, (148 * 4 if P == 1 else 148) // -(-P // 32))
    for lo in (0, max(0, N - few)):
        cut = slice(lo, lo + few)
        part, got = run(x[cut], r[cut] if residual else None, [u[cut] for u in ups])
        assert torch.equal(part.y, o.y[cut]) and torch.equal(got[0], grads[0][cut])
        rows = slice(lo, lo + few) if P == 1 else slice(lo * C, (lo + few) * C)
        assert torch.equal(part.q8.codes, o.q8.codes[rows]) and torch.equal(part.q8.scales, o.q8.scales[rows])
    assert (o.q8.codes[:, C if P == 1 else P:] == 0).all()


@pytest.mark.parametrize("N,C,P", [(5, 8, (1 << 26) + 32), (4, 9, (1 << 26) + 5), (70003, 32768, 1)])
def test_more_than_2_31_values(N, C, P):
    """Images (rows) whose offsets leave 32 bits: the last one is what it is alone."""
    shape = (N, C) if P == 1 else (N, C, P)
    last = slice(N - 1, N)
    gen = torch.Generator("cuda").manual_seed(1)
    make = lambda: torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    x, r, gy, gs = make().requires_grad_(True), make().requires_grad_(True), make(), make()
    w = (1 + 0.3 * torch.randn(C, device="cuda", generator=gen)).requires_grad_(True)
    o = tnn.rms_norm(x, w, r, output="both")
    gx, gr = torch.autograd.grad((o.y, o.stream), (x, r), (gy, gs))
    xs, rs = x[last].detach().requires_grad_(True), r[last].detach().requires_grad_(True)
    a = tnn.rms_norm(xs, w, rs, output="both")
    ax, _ = torch.autograd.grad((a.y, a.stream), (xs, rs), (gy[last], gs[last]))
    assert torch.equal(o.y[last], a.y) and torch.equal(o.stream[last], a.stream) and torch.equal(gx[last], ax)
    rows = a.q8.codes.shape[0]
    assert torch.equal(o.q8.codes[-rows:], a.q8.codes) and torch.equal(o.q8.scales[-rows:], a.q8.scales)


@pytest.mark.parametrize("C,P", [(17, (1 << 26) + 32), (33, (1 << 26) + 5)])
def test_images_of_more_than_2_30_values(C, P):
    """The kernels in groups where offsets inside an image leave 32 bits: the last positions against a short signal of them alone,
    to the roundings of both."""
    gen = torch.Generator("cuda").manual_seed(2)
    make = lambda: torch.empty(1, C, P, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    x, gy = make().requires_grad_(True), make()
    w = (1 + 0.3 * torch.randn(C, device="cuda", generator=gen)).requires_grad_(True)
    o = tnn.rms_norm(x, w, output="both", checkpoint="q8")
    (gx,) = torch.autograd.grad(o.y, x, gy)
    lo = P // 32 * 32 - 640                              # a border of the 8-bit blocks
    xs = x[..., lo:].detach().contiguous().requires_grad_(True)
    a = tnn.rms_norm(xs, w, output="both", checkpoint="q8")
    (ax,) = torch.autograd.grad(a.y, xs, gy[..., lo:].contiguous())
    s = _np(xs)
    want = ref.norm(s, _np(w), 1e-6, _np(gy[..., lo:]), None, True, "bf16")
    for got, name in ((o.y[..., lo:], "y"), (gx[..., lo:], "grad_x"), (a.y, "y"), (ax, "grad_x")):
        ref.check(_np(got), want[name], name)
    part = tnn.Q8(o.q8.codes[:, lo:].contiguous(), o.q8.scales[:, lo // 32:].contiguous(), xs.shape, xs.dtype)
    _q8_close(part, want["y32"], C, P - lo, "q8")
