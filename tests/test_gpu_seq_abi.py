"""The C entry points of the sequence and storage operators through their ctypes binding: what they write stays inside their
buffers, is what the torch functions give, and pointers that may be NULL may."""
import numpy as np
import pytest
import torch

from paper_2504_06881_b200 import nn as tnn, tconv, tseq
from test_gpu_guard_bands import Arena

pytestmark = pytest.mark.gpu
DT = tconv.TORCH_DTYPE
SIZE = {"f32": 4, "bf16": 2}


def _ok(rc):
    assert rc == 0, tconv.tconv_status_string(rc)


def _q8_buffers(arena, rows, inner):
    return (arena.take(tseq.tconv_q8_codes_bytes(rows, inner), torch.int8, (rows, -1)),
            arena.take(tseq.tconv_q8_scales_bytes(rows, inner), torch.uint8, (rows, -1)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (2, 100), (5, 3, 7), (4, 3, 31), (2, 3, 32), (3, 5, 49), (2, 5, 260), (70, 90, 24), (9, 11, 33)])
def test_store_and_restore(shape, dtype):
    rows, inner = (shape[0] * shape[1], shape[2]) if len(shape) == 3 else shape
    x = torch.randn(shape, device="cuda").to(DT[dtype])
    want = tnn.q8_store(x)
    a = Arena(4 << 20)
    codes, scales = _q8_buffers(a, rows, inner)
    back = a.take(x.numel() * SIZE[dtype], DT[dtype], shape)
    _ok(tseq.tconv_q8_store(rows, inner, dtype, x, codes, scales))
    _ok(tseq.tconv_q8_restore(rows, inner, dtype, codes, scales, back))
    torch.cuda.synchronize()
    assert torch.equal(codes, want.codes) and torch.equal(scales, want.scales) and torch.equal(back, want.restore())
    a.check("store and restore")


# (N, C, L): several rows a warp, a warp a row, a block a row, parts of a row; rows of whole vectors and of odd length
SCANS = [(3, 5, 1), (2, 3, 8), (5, 3, 7), (7, 3, 31), (2, 3, 32), (3, 5, 100), (2, 7, 127), (40, 70, 264), (40, 70, 301), (4, 90, 2048), (4, 90, 2051),
         (1, 3, 20000), (2, 3, 20001), (60, 100, 520)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("N,C,L", SCANS)
def test_scan(N, C, L, packed, kept, dtype):
    dt, n = DT[dtype], N * C * L
    gen = torch.Generator("cuda").manual_seed(n)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    both = randn(N, 2 * C, L).to(dt)
    x, g = both[:, :C], both[:, C:]
    if not packed:
        x, g = x.contiguous(), g.contiguous()
    h0, gy, gh = randn(N, C), randn(N, C, L).to(dt), randn(N, C)
    lengths = torch.randint(0, L + 1, (N,), dtype=torch.int32, device="cuda", generator=gen)
    lengths[0] = L
    ins = [(both if packed else x).detach().requires_grad_(True)]
    gi = None if packed else g.detach().requires_grad_(True)
    hi = h0.detach().requires_grad_(True)
    y, last = tnn.gated_scan(ins[0], gi, hi, lengths, "q8" if kept else None)
    want = torch.autograd.grad((y, last), ins + ([] if packed else [gi]) + [hi], (gy, gh))
    wide = (2 if packed else 1) * C * L
    d = tseq.scan_desc(N, C, L, dtype, x.stride(0), x.stride(1), g.stride(0), g.stride(1), wide)
    a = Arena(n * 24 + (32 << 20))
    yb, lb = a.take(n * SIZE[dtype], dt, (N, C, L)), a.take(4 * N * C, torch.float32, (N, C))
    states = a.take(tseq.tconv_scan_states_bytes(d), torch.float32)
    q = _q8_buffers(a, N * C, L) + _q8_buffers(a, N * C, L) if kept else (None,) * 4
    nws = tseq.tconv_scan_workspace_bytes(d, False)
    ws = a.take(nws) if nws else None
    _ok(tseq.tconv_scan_forward(d, x, g, h0, lengths, yb, lb, states, q, ws))
    grads = a.take((2 if packed else 1) * n * SIZE[dtype], dt, (N, -1, L))
    if packed:                                            # halves of one tensor: the second starts C rows in
        gx, gg = grads[:, :C], grads[:, C:]
    else:
        gx, gg = grads, a.take(n * SIZE[dtype], dt, (N, C, L))
    gh0 = a.take(4 * N * C, torch.float32, (N, C))
    nws = tseq.tconv_scan_workspace_bytes(d, True)
    ws = a.take(nws) if nws else None
    args = (None if kept else x, None if kept else g, lengths, states, gy)
    _ok(tseq.tconv_scan_backward(d, *args, gh, gx, gg, gh0, q, ws))
    torch.cuda.synchronize()
    a.check("scan")
    assert torch.equal(yb, y) and torch.equal(lb, last) and torch.equal(gh0, want[-1])
    if kept:
        live = torch.arange(L, device="cuda") < lengths[:, None, None]
        for t, (codes, scales) in ((x, q[:2]), (g, q[2:])):
            s = tnn.q8_store(torch.where(live, t, torch.zeros_like(t)).reshape(1, N * C, L) if L > 1 else
                             torch.where(live, t, torch.zeros_like(t)).reshape(N * C, 1))
            assert torch.equal(codes, s.codes) and torch.equal(scales, s.scales)
    for got, t in zip((grads,) if packed else (gx, gg), want):
        assert torch.equal(got, t)
    # no first state and none wanted back, no gradient of the last one; nothing kept for a backward pass
    none = torch.zeros_like
    y0, l0 = none(yb), none(lb)
    _ok(tseq.tconv_scan_forward(d, x, g, None, None, y0, l0, None, (None,) * 4, ws))
    w0 = tnn.gated_scan(x, g)
    assert torch.equal(y0, w0[0]) and torch.equal(l0, w0[1])
    before = gh0.clone()
    _ok(tseq.tconv_scan_backward(d, *args, None, gx, gg, None, q, ws))
    y, last = tnn.gated_scan(ins[0], gi, hi, lengths, "q8" if kept else None)
    want = torch.autograd.grad(y, ins + ([] if packed else [gi]), gy)
    for got, t in zip((grads,) if packed else (gx, gg), want):
        assert torch.equal(got, t)
    assert torch.equal(gh0, before)
    a.check("scan without states")


# forms of the kernels by channels and positions: all in registers, in groups, rows of channels
NORMS = [(3, 7, 1), (2, 512, 1), (5, 33, 1), (3, 1028, 1), (2, 1025, 1), (700, 64, 1), (2, 16, 7), (3, 20, 31), (2, 64, 32), (2, 33, 33), (4, 12, 49),
         (3, 24, 12), (2, 100, 28), (3, 512, 49), (2, 200, 49), (2, 300, 24), (2, 513, 40), (2, 513, 41), (2, 516, 12), (1, 8200, 33), (600, 20, 20)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("N,C,L", NORMS)
def test_norm(N, C, L, kept, residual, dtype):
    dt, n = DT[dtype], N * C * L
    shape = (N, C, L) if L > 1 else (N, C)
    rows, inner = (N * C, L) if L > 1 else (N, C)
    gen = torch.Generator("cuda").manual_seed(n)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    x, r = randn(*shape).to(dt), randn(*shape).to(dt) if residual else None
    gy, gs, w = randn(*shape).to(dt), randn(*shape).to(dt) if residual else None, 1 + 0.2 * randn(C)
    xi, wi, ri = x.detach().requires_grad_(True), w.detach().requires_grad_(True), r.detach().requires_grad_(True) if residual else None
    o = tnn.rms_norm(xi, wi, ri, 1e-5, "both", "q8" if kept else None)
    want = torch.autograd.grad([o.y] + [o.stream] * residual, [xi, wi], [gy] + [gs] * residual)
    d = tseq.norm_desc(N, C, L, dtype, 1e-5)
    a = Arena(n * 32 + (16 << 20))
    take = lambda: a.take(n * SIZE[dtype], dt, shape)
    s, y, rstd = take() if residual else None, take(), a.take(4 * N * L, torch.float32)
    yq, sq = _q8_buffers(a, rows, inner), _q8_buffers(a, rows, inner) if kept else (None, None)
    _ok(tseq.tconv_norm_forward(d, x, r, w, s, y, rstd, yq, sq))
    gx, gw = take(), a.take(4 * C, torch.float32)
    ws = a.take(tseq.tconv_norm_workspace_bytes(d))
    stream = None if kept else s if residual else x
    _ok(tseq.tconv_norm_backward(d, stream, rstd, w, gy, gs, gx, gw, sq, ws))
    torch.cuda.synchronize()
    a.check("norm")
    assert torch.equal(y, o.y) and (not residual or torch.equal(s, o.stream))
    assert torch.equal(yq[0], o.q8.codes) and torch.equal(yq[1], o.q8.scales)
    if kept:
        q = tnn.q8_store(o.stream.detach())
        assert torch.equal(sq[0], q.codes) and torch.equal(sq[1], q.scales)
    assert torch.equal(gx, want[0]) and torch.equal(gw, want[1])
    # y alone, its 8-bit form alone; no rstd, no gradient of the weight and then no workspace
    y2, q2, gx2 = take(), _q8_buffers(a, rows, inner), take()
    _ok(tseq.tconv_norm_forward(d, x, r, w, s, y2))
    _ok(tseq.tconv_norm_forward(d, x, r, w, s, None, None, q2))
    _ok(tseq.tconv_norm_backward(d, stream, rstd, w, gy, gs, gx2, None, sq))
    torch.cuda.synchronize()
    a.check("norm, fewer outputs")
    assert torch.equal(y2, y) and torch.equal(q2[0], yq[0]) and torch.equal(q2[1], yq[1]) and torch.equal(gx2, gx)
