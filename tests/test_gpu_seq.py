"""Gated scan, RMS norm and 8-bit store against their plain 64-bit forms (seq_ref)."""
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


def _scan_inputs(N, C, L, dtype, seed, spread=1.0):
    rs = np.random.RandomState(seed)
    x = rs.standard_normal((N, C, L))
    g = rs.standard_normal((N, C, L)) * spread + rs.uniform(-2, 5, (1, C, 1))
    return _t(x, dtype, True), _t(g, dtype, True), _t(rs.standard_normal((N, C)), grad=True), \
        _t(rs.standard_normal((N, C, L)), dtype), _t(rs.standard_normal((N, C)))


def _check_scan(x, g, h0, lengths, gy, gh, dtype, checkpoint, packed=False):
    want = ref.scan(_np(x), _np(g), None if h0 is None else _np(h0), None if lengths is None else lengths.cpu().numpy(), _np(gy),
                    _np(gh), checkpoint == "q8", dtype)
    if packed:
        both = torch.cat([x, g], 1).detach().requires_grad_(True)
        y, last = tnn.gated_scan(both, h0=h0, lengths=lengths, checkpoint=checkpoint)
        (gb, *rest) = torch.autograd.grad((y, last), [both] + ([] if h0 is None else [h0]), (gy, gh))
        gx, gg = gb.chunk(2, 1)
    else:
        y, last = tnn.gated_scan(x, g, h0, lengths, checkpoint)
        gx, gg, *rest = torch.autograd.grad((y, last), [x, g] + ([] if h0 is None else [h0]), (gy, gh))
    for name, t in (("y", y), ("h_last", last), ("grad_x", gx), ("grad_gate", gg)) + ((("grad_h0", rest[0]),) if rest else ()):
        assert t.dtype == (DT[dtype] if name in ("y", "grad_x", "grad_gate") else torch.float32)
        ref.check(_np(t), want[name], name)
    # without recording the same outputs, bit for bit
    with torch.no_grad():
        y2, last2 = tnn.gated_scan(x, g, h0, lengths)
    assert torch.equal(y, y2) and torch.equal(last, last2)


LENGTHS = [1, 2, 3, 7, 8, 9, 16, 31, 32, 33, 63, 64, 65, 127, 129, 255, 256, 257, 300, 511, 513, 1000, 2047, 2049, 4097]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("L", LENGTHS)
def test_scan_lengths(L, checkpoint, dtype):
    N, C = (3, 5) if L < 1000 else (2, 3)
    x, g, h0, gy, gh = _scan_inputs(N, C, L, dtype, L)
    _check_scan(x, g, h0, None, gy, gh, dtype, checkpoint)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("N,C,L", [(1, 1, 1), (1, 1, 20011), (1, 2, 16384), (2, 3, 6000), (70, 130, 40), (300, 33, 8), (9, 500, 264),
                                   (513, 1, 17), (40, 64, 512)])
def test_scan_shapes(N, C, L, checkpoint, dtype):
    """Few rows and long, many and short: whatever way the rows are split."""
    x, g, h0, gy, gh = _scan_inputs(N, C, L, dtype, N + C + L)
    _check_scan(x, g, h0, None, gy, gh, dtype, checkpoint)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("L", [1, 5, 40, 260, 777, 2048, 9001])
def test_scan_ragged(L, checkpoint, dtype):
    """Lengths of zero, one, all, and beyond both ends (held to 0..L); what lies behind a length is never used."""
    x, g, h0, gy, gh = _scan_inputs(7, 3, L, dtype, L)
    lengths = torch.tensor([0, 1, L, L // 2, max(L - 1, 0), L + 9, -3], dtype=torch.int32, device="cuda")
    with torch.no_grad():
        for n, m in enumerate([0, 1, L, L // 2, max(L - 1, 0), L, 0]):
            for t, bad in ((x, float("nan")), (g, float("inf")), (gy, float("nan"))):
                t[n, :, m:] = bad
    clean = [t.detach().nan_to_num(0, 0, 0) for t in (x, g, gy)]
    _check_scan(x, g, h0, lengths, gy, gh, dtype, checkpoint)
    y, last = tnn.gated_scan(x, g, h0, lengths, checkpoint)
    y2, last2 = tnn.gated_scan(clean[0], clean[1], h0.detach(), lengths.long())
    assert torch.equal(y, y2) and torch.equal(last, last2)
    assert (y[0] == 0).all() and torch.equal(last[0], h0[0]) and torch.equal(last[6], h0[6])
    # the same masking with the state absent
    _check_scan(x, g, None, lengths, gy, gh, dtype, checkpoint)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("L", [1, 24, 37, 512, 1021])
def test_scan_packed_and_strided(L, checkpoint, dtype):
    x, g, h0, gy, gh = _scan_inputs(3, 5, L, dtype, L + 3)
    _check_scan(x, g, h0, None, gy, gh, dtype, checkpoint, packed=True)
    # parts of a longer signal, every second channel, a broadcast batch, channels last
    y, last = tnn.gated_scan(x, g, h0)
    wide = torch.randn(3, 10, L + 13, device="cuda").to(DT[dtype])
    xs, gs = wide[:, ::2, 3:3 + L], wide[:, 1::2, 5:5 + L]
    xs.copy_(x.detach())
    gs.copy_(g.detach())
    xs, gs = xs.requires_grad_(True), gs.requires_grad_(True)
    ys, lasts = tnn.gated_scan(xs, gs, h0, checkpoint=checkpoint)
    assert torch.equal(y, ys) and torch.equal(last, lasts)
    a = torch.autograd.grad((ys, lasts), (xs, gs), (gy, gh))
    yc, lc = tnn.gated_scan(x, g, h0, checkpoint=checkpoint)
    b = torch.autograd.grad((yc, lc), (x, g), (gy, gh))
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    tl = x.detach().transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(tnn.gated_scan(tl, g.detach(), h0.detach())[0], y)
    one = x.detach()[:1].expand(3, -1, -1)
    assert torch.equal(tnn.gated_scan(one, g.detach(), h0.detach())[0], tnn.gated_scan(one.contiguous(), g.detach(), h0.detach())[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_extreme_gates_and_values(dtype):
    """Gates at both ends of the type: open (the state stays) and shut (the input passes); NaN and infinities reach what
    depends on them and nothing before them, nor other rows."""
    L = 700
    big = 3e38
    g = np.tile(np.array([big, -big, 200, -200, 90, -90, 0.0]), 100)[None, None, :].repeat(2, 1)
    x = np.random.RandomState(0).standard_normal((1, 2, L))
    xs, gs = _t(x, dtype), _t(g, dtype)
    y, last = tnn.gated_scan(xs, gs)
    ref.check(_np(y), ref.scan(_np(xs), _np(gs), dtype=dtype)["y"], "y")
    for bad, where in ((float("nan"), "x"), (float("inf"), "x"), (float("nan"), "g")):
        xb, gb = xs.clone(), torch.zeros_like(gs)
        (xb if where == "x" else gb)[0, 1, 300] = bad
        clean = tnn.gated_scan(xs, torch.zeros_like(gs))[0]
        yb, _ = tnn.gated_scan(xb, gb)
        assert torch.equal(yb[0, 0], clean[0, 0]) and torch.equal(yb[0, 1, :300], clean[0, 1, :300])
        assert not torch.isfinite(yb[0, 1, 300:400]).any()
        # kept in 8 bits: the block of the bad value, and what depends on it, is lost, other rows are not
        xq, gq = xb.clone().requires_grad_(True), gb.clone().requires_grad_(True)
        yq, _ = tnn.gated_scan(xq, gq, checkpoint="q8")
        assert torch.equal(yq[0, 0], clean[0, 0])
        gx, gg = torch.autograd.grad(yq, (xq, gq), torch.ones_like(yq))
        assert torch.isfinite(gx[0, 0]).all() and torch.isfinite(gg[0, 0]).all() and not torch.isfinite(gg[0, 1, 300])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_in_parts_and_steps(dtype):
    """A signal in one pass, in parts that hand the state on, and position by position."""
    x, g, h0, _, _ = _scan_inputs(3, 6, 50, dtype, 5)
    with torch.no_grad():
        y, last = tnn.gated_scan(x, g, h0)
        want = ref.scan(_np(x), _np(g), _np(h0), dtype=dtype)
        h, parts = h0, []
        for lo, hi in ((0, 1), (1, 9), (9, 33), (33, 50)):
            part, h = tnn.gated_scan(x[..., lo:hi], g[..., lo:hi], h)
            parts.append(part)
        ref.check(_np(torch.cat(parts, -1)), want["y"], "parts")
        ref.check(_np(h), want["h_last"], "parts")
        h, parts = h0.detach().clone(), []
        both = torch.cat([x, g], 1)
        for t in range(50):
            if t % 2:
                o, same = tnn.gated_scan_step(h, x[..., t], g[..., t], out=h)
                assert same.data_ptr() == h.data_ptr()
            else:
                before = h.clone()
                o, new = tnn.gated_scan_step(h, both[..., t].contiguous())
                assert torch.equal(h, before)
                h = new.clone()
            parts.append(o)
        ref.check(_np(torch.stack(parts, -1)), want["y"], "steps")
        ref.check(_np(h), want["h_last"], "steps")
    with pytest.raises(ValueError, match="records no gradients"):
        tnn.gated_scan_step(h0, x[..., 0], g[..., 0])
    with pytest.raises(ValueError, match="overlaps"), torch.no_grad():
        buf = torch.zeros(40, device="cuda")
        tnn.gated_scan_step(buf[:18].view(3, 6), x[..., 0], g[..., 0], out=buf[4:22].view(3, 6))


def test_scan_gradient_against_differences():
    """The directional derivative by differences of the 64-bit forward."""
    x, g, h0, gy, gh = _scan_inputs(2, 3, 70, "f32", 9)
    y, last = tnn.gated_scan(x, g, h0)
    grads = torch.autograd.grad((y, last), (x, g, h0), (gy, gh))
    rs = np.random.RandomState(1)
    base = [_np(t) for t in (x, g, h0)]
    for k in range(3):
        v = [rs.standard_normal(b.shape) if j == k else np.zeros(b.shape) for j, b in enumerate(base)]

        def loss(s):
            r = ref.scan(*(b + s * w for b, w in zip(base, v)))
            return (r["y"][0] * _np(gy)).sum() + (r["h_last"][0] * _np(gh)).sum()

        num = (loss(1e-5) - loss(-1e-5)) / 2e-5
        got = (_np(grads[k]) * v[k]).sum()
        assert abs(got - num) <= 1e-5 * np.abs(_np(grads[k]) * v[k]).sum() + 1e-7


def test_scan_one_output_used():
    x, g, h0, gy, gh = _scan_inputs(2, 3, 300, "f32", 4)
    zero = torch.zeros_like
    for pick, ups in ((0, (gy, zero(gh))), (1, (zero(gy), gh))):
        a = torch.autograd.grad(tnn.gated_scan(x, g, h0)[pick], (x, g, h0), ups[pick])
        b = torch.autograd.grad(tnn.gated_scan(x, g, h0), (x, g, h0), ups)
        assert all(torch.equal(u, v) for u, v in zip(a, b))
    xg = x.detach()
    only = torch.autograd.grad(tnn.gated_scan(xg, g)[0], g, gy)[0]
    assert torch.equal(only, torch.autograd.grad(tnn.gated_scan(x, g)[0], g, gy)[0])


def test_long_offsets():
    """More than 2^31 values: the last rows are those of a small call."""
    N, C, L = 2, 5, 220_000_007
    x = torch.empty(N, C, L, dtype=torch.bfloat16, device="cuda")
    x.normal_(generator=torch.Generator("cuda").manual_seed(0))
    with torch.no_grad():
        y, last = tnn.gated_scan(x, x)
        for n, c in ((0, 0), (1, 4)):
            ys, ls = tnn.gated_scan(x[n:n + 1, c:c + 1], x[n:n + 1, c:c + 1])
            assert (y[n, c] - ys[0, 0]).abs().max() <= 2.0 ** -7 and (last[n, c] - ls[0, 0]).abs() <= 1e-5
    del y
    q = tnn.q8_store(x)
    back = q.restore()
    part = tnn.q8_store(x[1:, 4:].contiguous()).restore()
    assert torch.equal(back[1:, 4:], part)


# ---- 8-bit store ---------------------------------------------------------------------------------------------
SHAPES = [(1,), (7,), (100,), (1, 1), (3, 5), (2, 512), (5, 33), (2, 3, 1), (2, 3, 7), (4, 5, 31), (2, 3, 32), (3, 4, 33), (2, 9, 49),
          (1, 7, 250), (2, 3, 4, 5), (2, 3, 32, 32), (6, 5, 7, 7), (1, 2, 3, 5, 7), (2, 1, 8, 8, 8), (3, 2, 1, 1), (70, 90, 24)]


def _rows(shape):
    inner = int(np.prod(shape[2:], dtype=np.int64))
    return (1, shape[0]) if len(shape) == 1 else (shape[0] * shape[1], inner) if inner > 1 else (shape[0], shape[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_q8(shape, dtype):
    """Codes, scales and restored values exactly as defined, over magnitudes from below the smallest unit to the largest
    finite, borders of the scale rule, zeros of both signs, infinities and NaN."""
    rs = np.random.RandomState(len(shape) + sum(shape))
    rows, inner = _rows(shape)
    v = rs.standard_normal(shape) * 2.0 ** rs.randint(-140, 120, shape[:1] + (1,) * (len(shape) - 1)).astype(np.float64)
    flat = v.reshape(-1)
    special = [0.0, -0.0, 127.5, 127.25, 127.0, 1.9921875, 1.984375, 2.0 ** -126, 2.0 ** -133, 3.3e38, -1.0, 0.5, 1.5, 2.5]
    at = rs.permutation(flat.size)[:max(1, flat.size // 40)]
    flat[at] = rs.choice(special, at.size)
    if flat.size > 300:
        flat[rs.permutation(flat.size)[:3]] = [np.nan, np.inf, -np.inf]
    x = _t(v, dtype)
    codes, scales, vals = ref.q8(_np(x), rows, inner)
    q = tnn.q8_store(x)
    assert q.codes.shape == (rows, (inner + 7) // 8 * 8) and q.codes.dtype == torch.int8 and q.scales.dtype == torch.uint8
    got = q.codes.cpu().numpy()
    assert np.array_equal(got[:, :inner], codes) and (got[:, inner:] == 0).all()
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    for dt in (None, torch.float32, torch.bfloat16):
        back = q.restore(dt)
        assert back.shape == x.shape and back.dtype == (dt or x.dtype)
        assert np.array_equal(_np(back).reshape(rows, inner), vals, equal_nan=True)
    if len(shape) > 1:                      # another order in memory
        xt = x.transpose(0, -1).contiguous().transpose(0, -1)
        assert torch.equal(tnn.q8_store(xt).codes, q.codes)


# ---- norm ----------------------------------------------------------------------------------------------------
def _q8_close(q, y32, rows, inner, what):
    """Codes and scales of a value known up to a bound: the scale is the one rule's for some value within it, and every
    restored value within half a unit and the bound."""
    val, bound = (a.reshape(rows, inner) for a in y32)
    units = 2.0 ** (q.scales.cpu().numpy().astype(np.float64) - 127)
    pad = -(-inner // 32) * 32 - inner
    blocks = lambda a: np.pad(a, ((0, 0), (0, pad))).reshape(rows, -1, 32).max(2)
    assert (blocks(np.abs(val) - bound) < 127.5 * units).all(), what
    big = blocks(np.abs(val) + bound)
    assert ((big >= 127.5 * units / 2) | (units == 2.0 ** -126)).all(), what
    back = _np(q.restore(torch.float32)).reshape(rows, inner)
    assert (np.abs(back - val) <= 0.5 * np.repeat(units, 32, 1)[:, :inner] * (1 + 1e-6) + bound).all(), what


NORM_SHAPES = [(1, 1), (3, 7), (2, 512), (5, 33), (1, 1000), (700, 64), (2, 5, 1), (1, 1, 2), (2, 3, 3), (2, 16, 7), (3, 20, 31), (2, 64, 32),
               (2, 33, 33), (4, 12, 49), (1, 5, 64), (2, 31, 65), (2, 128, 200), (1, 300, 96), (2, 513, 40), (1, 1030, 17), (2, 64, 8, 8),
               (3, 512, 7, 7), (2, 10, 4, 5, 6), (1, 256, 16, 32), (1, 4, 3981)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("checkpoint", [None, "q8"])
@pytest.mark.parametrize("shape", NORM_SHAPES)
def test_norm(shape, checkpoint, residual, dtype):
    rs = np.random.RandomState(sum(shape))
    x, w = _t(rs.standard_normal(shape), dtype, True), _t(1 + 0.3 * rs.standard_normal(shape[1]), grad=True)
    r = _t(2 * rs.standard_normal(shape), dtype, True) if residual else None
    gy, gs = _t(rs.standard_normal(shape), dtype), _t(rs.standard_normal(shape), dtype)
    eps = 1e-5
    stream = (x.float() + r.float()).to(DT[dtype]).detach() if residual else x.detach()
    N, C = shape[:2]
    three = lambda t: _np(t).reshape(N, C, -1)
    want = ref.norm(three(stream), _np(w), eps, three(gy), three(gs) if residual else None, checkpoint == "q8", dtype)
    o = tnn.rms_norm(x, w, r, eps, output="both", checkpoint=checkpoint)
    assert torch.equal(o.stream, stream)
    ref.check(three(o.y), want["y"], "y")
    _q8_close(o.q8, want["y32"], *_rows(shape), "q8")
    ins, outs, ups = ([x, w, r], [o.y, o.stream], [gy, gs]) if residual else ([x, w], [o.y], [gy])
    grads = torch.autograd.grad(outs, ins, ups)
    ref.check(three(grads[0]), want["grad_x"], "grad_x")
    ref.check(_np(grads[1]), want["grad_weight"], "grad_weight")
    if residual:
        assert torch.equal(grads[0], grads[2])
        # the stream alone, y alone
        only = torch.autograd.grad(tnn.rms_norm(x, w, r, eps).stream, (x, r), gs)
        ref.check(_np(only[0]), (_np(gs), np.zeros(shape)), "stream alone")
        alone = ref.norm(three(stream), _np(w), eps, three(gy), None, checkpoint == "q8", dtype)
        gx = torch.autograd.grad(tnn.rms_norm(x, w, r, eps, checkpoint=checkpoint).y, x, gy)[0]
        ref.check(three(gx), alone["grad_x"], "y alone")
    with torch.no_grad():                    # the other outputs, not recorded
        for output in ("same", "both", "q8"):
            p = tnn.rms_norm(x, w, r, eps, output=output)
            assert (p.y is None) == (output == "q8") and (p.q8 is None) == (output == "same")
            assert p.y is None or torch.equal(p.y, o.y)
            assert p.q8 is None or (torch.equal(p.q8.codes, o.q8.codes) and torch.equal(p.q8.scales, o.q8.scales))
            assert torch.equal(p.stream, stream)
    with pytest.raises(ValueError, match="nothing to differentiate"):
        tnn.rms_norm(x, w, r, output="q8")


def test_norm_gradient_against_differences():
    rs = np.random.RandomState(3)
    x, w = rs.standard_normal((2, 9, 11)), 1 + 0.3 * rs.standard_normal(9)
    gy = rs.standard_normal(x.shape)
    xt, wt = _t(x, grad=True), _t(w, grad=True)
    gx, gw = torch.autograd.grad(tnn.rms_norm(xt, wt).y, (xt, wt), _t(gy))
    x, w, gy = _np(xt), _np(wt), _np(_t(gy))
    for got, d in ((gx, (1, 0)), (gw, (0, 1))):
        v = rs.standard_normal(got.shape)
        loss = lambda s: (ref.norm(x + d[0] * s * (v if d[0] else 0), w + d[1] * s * (v if d[1] else 0))["y"][0] * gy).sum()
        num = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert abs((_np(got) * v).sum() - num) <= 1e-5 * np.abs(_np(got) * v).sum() + 1e-7


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 40), (2, 40, 70), (2, 64, 64)])
def test_norm_special_values(shape, dtype):
    """A row of zeros stays zero; a NaN or an infinity reaches its own position's channels only."""
    x = _t(np.random.RandomState(0).standard_normal(shape), dtype)
    w = torch.ones(shape[1], device="cuda")
    clean = tnn.rms_norm(x, w).y
    z = x.clone()
    z[0] = 0
    y = tnn.rms_norm(z, w, output="both")
    assert (y.y[0] == 0).all() and (y.q8.codes[:1] == 0).all() and torch.equal(y.y[1], clean[1])
    for bad in (float("nan"), float("inf")):
        b = x.clone()
        at = (1, 3) + (5,) * (len(shape) - 2)
        b[at] = bad
        y = tnn.rms_norm(b, w).y
        hit = torch.zeros(shape, dtype=torch.bool, device="cuda")
        hit[(1, slice(None)) + at[2:]] = True
        assert torch.equal(y[~hit], clean[~hit])
        assert torch.isnan(y[at]) and (torch.isnan(y[hit]) | (y[hit] == 0)).all()


# ---- how they are called -------------------------------------------------------------------------------------
def _everything(t):
    """Outputs and gradients of one pass through all three."""
    y, last = tnn.gated_scan(t["x"], t["g"], t["h0"], checkpoint=t["ck"])
    o = tnn.rms_norm(y, t["w"], t["r"], output="both", checkpoint=t["ck"])
    grads = torch.autograd.grad((o.y, o.stream, last), (t["x"], t["g"], t["h0"], t["w"], t["r"]), (t["gy"], t["gs"], t["gh"]))
    return [o.y.detach(), o.stream.detach(), last.detach(), o.q8.codes, o.q8.scales, o.q8.restore(), *grads]


def _tensors(N, C, L, dtype, ck, seed):
    x, g, h0, gy, gh = _scan_inputs(N, C, L, dtype, seed)
    rs = np.random.RandomState(seed + 1)
    return dict(x=x, g=g, h0=h0, gy=gy, gh=gh, w=_t(1 + 0.1 * rs.standard_normal(C), grad=True),
                r=_t(rs.standard_normal((N, C, L)), dtype, True), gs=_t(rs.standard_normal((N, C, L)), dtype), ck=ck)


CALLS = [(2, 8, 1000, "f32", None), (1, 3, 30000, "bf16", "q8"), (2, 33, 49, "bf16", None), (64, 48, 1, "f32", "q8"), (1, 2, 20001, "f32", None)]


@pytest.mark.parametrize("N,C,L,dtype,ck", CALLS)
def test_calls_repeat_bit_for_bit_on_any_stream(N, C, L, dtype, ck):
    t = _tensors(N, C, L, dtype, ck, 3)
    want = _everything(t)
    assert all(torch.equal(a, b) for a, b in zip(want, _everything(t)))
    other = _tensors(N, C, L, dtype, ck, 4)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for k in range(4):                       # two at once, several rounds
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                r = _everything((t, other)[i])
                if i == 0:
                    got.append(r)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in got for a, b in zip(want, r))


@pytest.mark.parametrize("N,C,L,dtype,ck", CALLS)
def test_captured_and_replayed(N, C, L, dtype, ck):
    """Forward and backward in a graph, replayed on other values; two graphs that share their memory pool replay in turn."""
    first, second = (_tensors(N, C, L, dtype, ck, s) for s in (5, 6))
    want = [_everything(first), _everything(second)]
    t = _tensors(N, C, L, dtype, ck, 5)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(2):
            _everything(t)
    torch.cuda.synchronize()
    pool = torch.cuda.graph_pool_handle()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool, stream=side):
            outs.append(_everything(t))
        graphs.append(graph)
    for turn, src in ((0, first), (1, second), (0, second), (1, first)):
        with torch.no_grad():
            for k, v in t.items():
                if isinstance(v, torch.Tensor):
                    v.copy_(src[k])
        graphs[turn].replay()
        torch.cuda.synchronize()
        ref_out = want[0 if src is first else 1]
        assert all(torch.equal(a, b) for a, b in zip(outs[turn], ref_out)), (turn, src is first)


def test_refusals_on_the_gpu():
    x = torch.zeros(2, 4, 8, device="cuda")
    h = torch.zeros(2, 4, device="cuda")
    w = torch.ones(4, device="cuda")
    for call in (lambda: tnn.gated_scan(x, x.bfloat16()), lambda: tnn.gated_scan(x.half(), x.half()), lambda: tnn.gated_scan(x[0], x[0]),
                 lambda: tnn.gated_scan(x, x[..., :4]), lambda: tnn.gated_scan(x[:, :3]), lambda: tnn.gated_scan(x, x, h.double()),
                 lambda: tnn.gated_scan(x, x, h[:1]), lambda: tnn.gated_scan(x, x, lengths=torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: tnn.gated_scan(x, x, lengths=torch.zeros(2, dtype=torch.int32)), lambda: tnn.gated_scan(x, x.cpu()),
                 lambda: tnn.gated_scan_step(h, x[..., 0], x[:, :2, 0]), lambda: tnn.gated_scan_step(h.bfloat16(), x[..., 0], x[..., 0]),
                 lambda: tnn.rms_norm(x, w[:3]), lambda: tnn.rms_norm(x, w.cpu()), lambda: tnn.rms_norm(x, w, x[:1]),
                 lambda: tnn.rms_norm(x, w, x.bfloat16()), lambda: tnn.rms_norm(x[0, 0], w), lambda: tnn.rms_norm(x.long(), w),
                 lambda: tnn.q8_store(x.half()), lambda: tnn.q8_store(torch.zeros((), device="cuda")),
                 lambda: tnn.Q8(torch.zeros(2, 8, dtype=torch.int8, device="cuda"), torch.zeros(2, 1, dtype=torch.uint8, device="cuda"),
                                (3, 8), torch.float32).restore()):
        with pytest.raises(ValueError):
            call()
    empty = torch.zeros(2, 4, 0, device="cuda")
    for call in (lambda: tnn.gated_scan(empty, empty), lambda: tnn.rms_norm(empty, w), lambda: tnn.q8_store(empty),
                 lambda: tnn.q8_store(x[:0]), lambda: tnn.rms_norm(x, w, eps=-1.0)):
        with pytest.raises(tconv.TconvError) as e:
            call()
        assert e.value.status == -1
    a = x.clone().requires_grad_(True)
    y, _ = tnn.gated_scan(a, a)
    with pytest.raises(NotImplementedError, match="second derivative"):
        torch.autograd.grad(y.sum(), a, create_graph=True)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y, _ = tnn.gated_scan(a, a)
        with torch.no_grad():
            a.add_(1)
        y.sum().backward()
    import torch.autograd.forward_ad as fwad
    with fwad.dual_level(), pytest.raises(NotImplementedError, match="forward-mode"):
        tnn.gated_scan(fwad.make_dual(x, x), x)
    with pytest.raises(NotImplementedError, match="traced"):
        torch.jit.trace(lambda v: tnn.rms_norm(v, w).y, x)
