"""The sequence and storage operators at the ends of their ranges."""
import numpy as np
import pytest
import torch

import seq_ref as ref
from paper_2504_06881_b200 import nn as tnn, tconv

pytestmark = pytest.mark.gpu
DT = tconv.TORCH_DTYPE


def _t(a, dtype="f32", grad=False):
    t = torch.from_numpy(np.asarray(a, np.float32)).to(DT[dtype]).cuda()
    return t.requires_grad_(True) if grad else t


def _np(t):
    return t.detach().double().cpu().numpy()


# ---- 8-bit form ----------------------------------------------------------------------------------------------
def _top_block(dtype):
    """Thirty-two values around the largest unit's border, both signs, small ones among them."""
    most = float(torch.finfo(DT[dtype]).max)
    unit = 2.0 ** 121
    return np.array([most, -most, 127.5 * unit, -127.5 * unit, 127 * unit, -127 * unit, 126.5 * unit, 125.5 * unit, 64 * unit, unit, -unit,
                     0.5 * unit, 1.5 * unit, 1.0, -1.0, 0.0] * 2)


def _top_values(v):
    """What such a block stands for: e = 121, codes held to 127."""
    unit = 2.0 ** 121
    return np.clip(np.rint(v / unit), -127, 127) * unit


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 32), (3, 32), (2, 2, 32), (2, 3, 70), (1, 5, 49), (2, 7)])
def test_q8_largest_finite_values(shape, dtype):
    """Blocks up to the type's largest finite value restore to finite values, those from 127.5 * 2^121 on to 127 * 2^121."""
    v = np.resize(_top_block(dtype), shape)
    x = _t(v, dtype)
    v = _np(x)                                           # (bf16: as rounded)
    assert np.isfinite(v).all()
    q = tnn.q8_store(x)
    want = _top_values(v)                                # (every block has a value beyond 127.5 units in it)
    assert (q.scales == 248).all()
    for dt in (torch.float32, torch.bfloat16):
        back = _np(q.restore(dt))
        assert np.array_equal(back, want)
    off = np.abs(want - v) / 2.0 ** 121
    assert (off[np.abs(v) < 127.5 * 2.0 ** 121] <= 0.5).all() and (off < 1).all()
    for s in (1.0, -1.0):
        full = torch.full(shape, s * torch.finfo(DT[dtype]).max, dtype=DT[dtype], device="cuda")
        assert (tnn.q8_store(full).restore() == s * 127 * 2.0 ** 121).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [5, 20, 100, 300, 33])
def test_scan_keeps_the_largest_finite_values(L, dtype):
    """What the recurrence keeps of candidates and gates at the type's ends is finite: with gates of the type's largest and
    lowest value the gradients over the restored ones are those of fully open and shut gates."""
    most = torch.finfo(DT[dtype]).max
    rs = np.random.RandomState(L)
    x, gy = _t(rs.standard_normal((1, 3, L)), dtype, True), _t(rs.standard_normal((1, 3, L)), dtype)
    for s in (1, -1):
        g = torch.full((1, 3, L), s * most, dtype=DT[dtype], device="cuda", requires_grad=True)
        y, last = tnn.gated_scan(x, g, checkpoint="q8")
        gx, gg = torch.autograd.grad(y, (x, g), gy)
        assert torch.isfinite(gx).all() and (gg == 0).all()
        if s > 0:
            assert (gx == 0).all() and (y == 0).all()
        else:
            assert torch.equal(y, x)
    x = torch.full((1, 3, L), most, dtype=DT[dtype], device="cuda", requires_grad=True)
    g = torch.zeros_like(x).requires_grad_(True)
    y, last = tnn.gated_scan(x, g, checkpoint="q8")
    gx, gg = torch.autograd.grad(y, (x, g), gy * 1e-6)
    assert torch.isfinite(gx).all() and torch.isfinite(gg).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 40), (2, 1028), (2, 40, 33), (2, 40, 64), (1, 1030, 40)])
def test_norm_stores_the_largest_finite_values(shape, dtype):
    """A weight of the largest finite value over a stream of ones: the 8-bit output is finite."""
    x = torch.ones(shape, dtype=DT[dtype], device="cuda")
    w = torch.full(shape[1:2], 3.4e38, device="cuda")
    o = tnn.rms_norm(x, w, eps=0.0, output="both")
    assert (o.q8.restore() == 127 * 2.0 ** 121).all() and (o.q8.scales == 248).all()


# ---- gates ---------------------------------------------------------------------------------------------------
EPS = ref.EPS
LENGTHS = [1, 2, 8, 9, 33, 128, 129, 300, 3000]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", LENGTHS)
def test_scan_shut_gates_and_large_states(L, dtype):
    """A first state of any size behind a gate that is nearly or fully shut, then gates of 0.  f is the sigmoid down to 2^-126 and
    zero below; e^-|g| is off by some (3 + |g|) steps of fp32 (the argument's rounding is |g| EPS, ex2 4 EPS), its sum, reciprocal and
    product by 5 EPS more."""
    most = float(torch.finfo(DT[dtype]).max)
    gates = [-most, -200.0, -104.0, -88.0, -87.0, -85.0, -80.0, -79.0, -60.0, -10.0]
    heights = [1.0, -1e30, 1e38, -3e38]
    G, H = (a.reshape(1, -1) for a in np.meshgrid(gates, heights))
    g = np.zeros((1, G.size, L))
    g[..., 0] = G
    gt, xt, h0 = _t(g, dtype), torch.ones(1, G.size, L, dtype=DT[dtype], device="cuda"), _t(H)
    y, last = tnn.gated_scan(xt, gt, h0)
    gv, hv = _np(gt)[..., 0], _np(h0)
    e = np.exp(gv)
    f = np.where(e / (1 + e) < 2.0 ** -126, 0.0, e / (1 + e))
    h = f * hv + (1 - f)
    off = np.abs(f * hv) * (2 * np.abs(np.where(f > 0, gv, 0.0)) + 12) * EPS + 8 * EPS * (np.abs(h) + 1)
    for t in range(min(L, 40)):
        if t:                                             # halving: exact gates, a few roundings
            h, off = h / 2 + 0.5, off / 2 + 8 * EPS * (np.abs(h) + 1)
        got = _np(y)[..., t]
        assert (np.abs(got - h) <= off + ref.HALF[dtype] * (np.abs(h) + off)).all(), t
    # a gate that is fully shut forgets: the same, bit for bit, from any state
    shut = torch.full_like(gt, 0.0)
    shut[..., L // 2] = -most
    xr = _t(np.random.RandomState(L).standard_normal((1, G.size, L)), dtype)
    a, la = tnn.gated_scan(xr, shut, h0)
    b, lb = tnn.gated_scan(xr, shut, torch.zeros_like(h0))
    shut[..., L // 2] = float("-inf")
    c, lc = tnn.gated_scan(xr, shut, h0)
    assert torch.equal(a[..., L // 2:], b[..., L // 2:]) and torch.equal(la, lb)
    assert torch.equal(c, a) and torch.equal(lc, la) and torch.equal(a[..., L // 2], xr[..., L // 2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("L", LENGTHS)
def test_scan_gradients_at_extreme_gates(L, checkpoint, dtype):
    """Rows cut by fully shut gates into stretches of three: gradients stay inside a stretch, and a shut gate has none of its own;
    rows that are open throughout: y is the first state, x has no gradient and h0 has all of it."""
    most = float(torch.finfo(DT[dtype]).max)
    rs = np.random.RandomState(L)
    x, gy = rs.standard_normal((2, 4, L)), rs.standard_normal((2, 4, L))
    g = np.zeros((2, 4, L))
    g[0, :, ::3] = -most if checkpoint else -np.inf
    g[1] = most if checkpoint else np.inf                 # (kept in 8 bits an infinity poisons its block)
    xt, gt, ht, gyt = _t(x, dtype, True), _t(g, dtype, True), _t(rs.standard_normal((2, 4)), grad=True), _t(gy, dtype)
    y, last = tnn.gated_scan(xt, gt, ht, checkpoint=checkpoint)
    gx, gg, gh = torch.autograd.grad(y, (xt, gt, ht), gyt)
    assert torch.equal(y[1], ht[1, :, None].expand_as(y[1]).to(y.dtype)) and torch.equal(last[1], ht[1])
    assert (gx[1] == 0).all() and (gg[1] == 0).all()
    total = _np(gyt)[1].sum(-1)
    assert (np.abs(_np(gh)[1] - total) <= (L + 8) * EPS * np.abs(_np(gyt)[1]).sum(-1)).all()
    assert (gh[0] == 0).all() and (gg[0, :, ::3] == 0).all()
    # D_t = dy_t + D_{t+1} / 2 inside a stretch; u is 1 at its start and 1/2 behind
    dy, D = _np(gyt)[0], np.zeros((4, L))
    for t in range(L - 1, -1, -1):
        D[:, t] = dy[:, t] + (0.5 * D[:, t + 1] if t + 1 < L and (t + 1) % 3 else 0.0)
    want = np.where(np.arange(L) % 3, 0.5, 1.0) * D
    assert (np.abs(_np(gx)[0] - want) <= (16 * EPS + ref.HALF[dtype]) * (np.abs(want) + 4 * np.abs(dy).max())).all()
    if dtype == "f32" and checkpoint is None:             # whatever lies in front of a stretch
        x2 = xt.detach().clone()
        x2[0, :, :3] = 1e30
        x2.requires_grad_(True)
        y2, _ = tnn.gated_scan(x2, gt, ht)
        g2 = torch.autograd.grad(y2, (x2, gt), gyt)
        assert torch.equal(y2[0, :, 3:], y[0, :, 3:]) and torch.equal(g2[0], gx) and torch.equal(g2[1][0, :, 3:], gg[0, :, 3:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,L", [(1, 400001), (16, 8192), (200, 8192)])
def test_scan_holds_a_constant(N, L, dtype):
    """Constant candidates x from the state h0 = x under constant gates that hardly decay: h stays x but for roundings that come
    back every step.  With f + u = 1 to half a step below 1, 2^-25 = EPS / 2, the fixed point u x / (1 - f) is off by EPS / 2u of x.
    The decay of 256 positions is a product of 256 factors below 1: 255 roundings of EPS / 2 in whatever order, at worst all one way
    since all are alike, EPS / 2u more; joining chunks and parts, and adding the state, take less than four roundings a chunk
    (4 / 256 EPS / u).  Sums of candidates err by EPS of themselves ten times or so, and a position by some ten roundings of its own.
    1.02 EPS / u + 20 EPS in all."""
    gates = np.repeat(np.linspace(8.0, 13.5, 24)[None], N, 0)
    g = _t(np.broadcast_to(gates[..., None], (N, 24, L)), dtype)
    x = torch.full((N, 24, L), 0.7, dtype=DT[dtype], device="cuda")
    h0 = x[..., 0].float()
    y, last = tnn.gated_scan(x, g, h0)
    u = 1 / (1 + np.exp(_np(g)[..., 0]))
    off = 1.02 * EPS / u + 20 * EPS
    err = np.abs(_np(last) / _np(h0) - 1)
    assert (err <= off).all(), (err / off).max()
    if dtype == "f32":
        top = (y / h0[..., None] - 1).abs().amax(-1)
        assert (_np(top) <= off + EPS).all(), (_np(top) / off).max()


@pytest.mark.parametrize("L", [1, 9, 33, 129, 300])
def test_scan_factors_add_up_to_one(L):
    """f is what a state of one becomes with candidates of zero, u what candidates of one make of no state: the larger of the two
    is 1 less the smaller, rounded once (EPS / 2), and the smaller within its own errors: e^-|g| to (|g| + 5) EPS, the sum, the
    reciprocal (2 EPS) and the product to 4 EPS."""
    g = np.concatenate([np.linspace(-80, 80, 4001), np.linspace(-14, 14, 20001), np.linspace(-0.1, 0.1, 2001)])
    gt = torch.zeros(1, g.size, L, device="cuda")
    gt[..., 0] = _t(g)
    zero, one = torch.zeros_like(gt), torch.ones(1, g.size, device="cuda")
    first = zero.clone()
    first[..., 0] = 1
    f, u = _np(tnn.gated_scan(zero, gt, one)[0])[0, :, 0], _np(tnn.gated_scan(first, gt)[0])[0, :, 0]
    assert (np.abs(f + u - 1) <= EPS / 2).all()
    gv = _np(gt)[0, :, 0]
    e = np.exp(-np.abs(gv))
    small, off = e / (1 + e), e / (1 + e) * (2 * np.abs(gv) + 9) * EPS
    for got, less in ((f, gv < 0), (u, gv >= 0)):
        want = np.where(less, small, 1 / (1 + e))
        assert (np.abs(got - want) <= off + np.where(less, 0, EPS / 2)).all()


# ---- gradients of one output, and the step -------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("shape", [(2, 40), (2, 33, 50), (2, 1030, 40)])
def test_norm_stream_alone_passes_its_gradient_on(shape, checkpoint, dtype):
    """Where only the stream is used its gradient is that of x and of the residual, whatever the stream holds; the weight's is 0."""
    rs = np.random.RandomState(1)
    x, r = _t(rs.standard_normal(shape), dtype), _t(rs.standard_normal(shape), dtype)
    x.view(-1)[3], x.view(-1)[77] = float("inf"), float("nan")
    w, up = torch.ones(shape[1], device="cuda", requires_grad=True), _t(rs.standard_normal(shape), dtype)
    x.requires_grad_(True)
    r.requires_grad_(True)
    s = tnn.rms_norm(x, w, r, checkpoint=checkpoint).stream
    gx, gw, gr = torch.autograd.grad(s, (x, w, r), up, retain_graph=True)
    assert torch.equal(gx, up) and torch.equal(gr, up) and (gw == 0).all() and gw.shape == w.shape
    (gx,) = torch.autograd.grad(s, (x,), up.transpose(0, 1).contiguous().transpose(0, 1))      # strided, and one wanted alone
    assert torch.equal(gx, up)
    # leaves have gradients of their own: not the caller's tensor, nor each other's
    tnn.rms_norm(x, w, r, checkpoint=checkpoint).stream.backward(up)
    assert torch.equal(x.grad, up) and torch.equal(r.grad, up) and (w.grad == 0).all()
    before = up.clone()
    x.grad.add_(1)
    assert torch.equal(r.grad, before) and torch.equal(up, before)


def test_step_refuses_a_state_that_overlaps_its_inputs():
    buf = torch.randn(64, device="cuda")
    h, x, g = torch.randn(2, 8, device="cuda"), torch.randn(2, 8, device="cuda"), torch.randn(2, 8, device="cuda")
    with torch.no_grad():
        want, state = tnn.gated_scan_step(h, x, g)
        for call in (lambda: tnn.gated_scan_step(h, buf[:16].view(2, 8), g, out=buf[4:20].view(2, 8)),
                     lambda: tnn.gated_scan_step(h, x, buf[16:32].view(2, 8), out=buf[4:20].view(2, 8)),
                     lambda: tnn.gated_scan_step(h, buf[:32].view(2, 16), out=buf[28:44].view(2, 8)),
                     lambda: tnn.gated_scan_step(h, buf[:64].view(8, 8)[::4], g, out=buf[24:40].view(2, 8))):
            with pytest.raises(ValueError, match="overlaps"):
                call()
        # neighbours are fine: next to each other, between the rows of a wider tensor; and the state itself
        buf.view(8, 8)[::4].copy_(x)
        y, out = tnn.gated_scan_step(h, buf.view(8, 8)[::4], g, out=buf[12:28].view(2, 8))
        assert torch.equal(y, want) and torch.equal(out, state) and torch.equal(buf.view(8, 8)[::4], x)
        buf[:16].copy_(x.view(-1))
        buf[16:32].copy_(g.view(-1))
        y, out = tnn.gated_scan_step(h, buf[:16].view(2, 8), buf[16:32].view(2, 8), out=buf[32:48].view(2, 8))
        assert torch.equal(y, want) and torch.equal(out, state)
        y, out = tnn.gated_scan_step(h, x, g, out=h)
        assert torch.equal(y, want) and torch.equal(out, state)


def test_step_and_store_refuse_tangents():
    import torch.autograd.forward_ad as fwad
    h, x, g = (torch.randn(2, 8, device="cuda") for _ in range(3))
    for k in range(3):
        with torch.no_grad(), fwad.dual_level(), pytest.raises(NotImplementedError, match="forward-mode"):
            t = [h, x, g]
            t[k] = fwad.make_dual(t[k], torch.ones_like(t[k]))
            tnn.gated_scan_step(*t)
    with fwad.dual_level(), pytest.raises(NotImplementedError, match="forward-mode"):
        tnn.q8_store(fwad.make_dual(x, torch.ones_like(x)))


@pytest.mark.parametrize("checkpoint", [None, "q8"])
def test_function_transforms_are_refused(checkpoint):
    """As the layers': what a transform hands over has no memory of its own."""
    x, g, h = torch.randn(2, 4, 8, device="cuda"), torch.randn(2, 4, 8, device="cuda"), torch.randn(2, 4, device="cuda")
    w, many = torch.ones(4, device="cuda"), lambda t: torch.stack([t, t])
    calls = [(lambda v: tnn.gated_scan(v, g, checkpoint=checkpoint)[0], x), (lambda v: tnn.gated_scan(x, v, checkpoint=checkpoint)[0], g),
             (lambda v: tnn.gated_scan(x, g, v, checkpoint=checkpoint)[0], h),
             (lambda v: tnn.rms_norm(v, w, checkpoint=checkpoint).y, x), (lambda v: tnn.rms_norm(x, v, checkpoint=checkpoint).y, w),
             (lambda v: tnn.rms_norm(x, w, v, checkpoint=checkpoint).y, x)]
    for fn, t in calls:
        for record in (True, False):
            with torch.set_grad_enabled(record), pytest.raises(RuntimeError):
                torch.func.vmap(fn)(many(t))
        with pytest.raises(RuntimeError):
            torch.func.grad(lambda v: fn(v).sum())(t)
    for fn, t in ((lambda v: tnn.q8_store(v).restore(), x), (lambda v: tnn.gated_scan_step(v, x[..., 0], g[..., 0])[0], h),
                  (lambda v: tnn.gated_scan_step(h, v, g[..., 0])[0], h),
                  (lambda v: tnn.gated_scan(x, g, lengths=v)[0], torch.tensor([3, 8], dtype=torch.int32, device="cuda"))):
        with pytest.raises(RuntimeError), torch.no_grad():
            torch.func.vmap(fn)(many(t))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("L", LENGTHS)
def test_scan_skips_lowest_values_behind_open_gates(L, checkpoint, dtype):
    """Positions masked by the type's lowest value and a fully open gate: the state passes them, they have no gradients, and all
    others are what they are with zeros there, bit for bit, under upstream gradients of any size."""
    most = float(torch.finfo(DT[dtype]).max)
    rs = np.random.RandomState(L)
    masked = torch.from_numpy(rs.rand(2, 5, L) < 0.3).cuda()
    masked[..., 0] = True
    x, g = _t(rs.standard_normal((2, 5, L)), dtype), _t(rs.standard_normal((2, 5, L)), dtype)
    h0, gy, gh = _t(rs.standard_normal((2, 5)), grad=True), _t(100 * rs.standard_normal((2, 5, L)), dtype), _t(rs.standard_normal((2, 5)))
    if checkpoint:                                        # whole rows of masks, alone in their 8-bit blocks
        masked[:] = False
        masked[1] = True
    g[masked] = most
    runs = []
    for value in (0.0, -most):
        xi, gi = torch.where(masked, value, x).to(DT[dtype]).requires_grad_(True), g.detach().requires_grad_(True)
        y, last = tnn.gated_scan(xi, gi, h0, checkpoint=checkpoint)
        runs.append((y, last) + torch.autograd.grad((y, last), (xi, gi, h0), (gy, gh)))
        assert all(torch.isfinite(t).all() for t in runs[-1])
        assert (runs[-1][2][masked] == 0).all() and (runs[-1][3][masked] == 0).all()
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("shape", [(2, 40), (2, 1028), (2, 40, 33), (2, 40, 64), (1, 520, 40)])
def test_norm_of_sums_beyond_fp32(shape, checkpoint, dtype):
    """A position whose squares leave fp32: y is 0 there, the gradient through the norm as well, and other positions are what they are;
    where a position lies in its neighbours' 8-bit blocks, theirs are not compared."""
    most = float(torch.finfo(DT[dtype]).max)
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(shape, device="cuda", generator=gen).to(DT[dtype])
    gy, gs = torch.randn(shape, device="cuda", generator=gen).to(DT[dtype]), torch.randn(shape, device="cuda", generator=gen).to(DT[dtype])
    r, w = torch.zeros_like(x), torch.ones(shape[1], device="cuda")

    def run(x):
        x = x.clone().requires_grad_(True)
        o = tnn.rms_norm(x, w, r, checkpoint=checkpoint)
        return (o.y.detach(),) + torch.autograd.grad((o.y, o.stream), x, (gy, gs))

    clean = run(x)
    at = (0, slice(None)) + (5,) * (len(shape) - 2)
    x[at][::2] = -most
    y, gx = run(x)
    assert (y[at] == 0).all() and torch.equal(gx[at], gs[at])
    other = torch.ones(shape, dtype=torch.bool, device="cuda")
    other[at] = False
    assert torch.equal(y[other], clean[0][other])
    if checkpoint and len(shape) > 2:
        other[0, :, :32] = False
    assert torch.equal(gx[other], clean[1][other])
