"""Sequence and storage operators: what the host refuses before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2504_06881_b200 import nn as tnn, tconv, tseq

P = ctypes.c_void_p


def _scan(d, **kw):
    a = dict(x=0x1000, gate=0x2000, h0=0, lengths=0, y=0x3000, h_last=0x4000, states=0x5000, xc=0, xs=0, gc=0, gs=0, ws=0)
    a.update(kw)
    return tconv._lib.tconv_scan_forward(ctypes.byref(d), *(P(v) for v in a.values()), 0, P(0))


def _scan_bwd(d, **kw):
    a = dict(x=0x1000, gate=0x2000, xc=0, xs=0, gc=0, gs=0, lengths=0, states=0x5000, gy=0x6000, gh=0, gx=0x7000, gg=0x8000,
             gh0=0, ws=0)
    a.update(kw)
    return tconv._lib.tconv_scan_backward(ctypes.byref(d), *(P(v) for v in a.values()), 0, P(0))


def test_q8_sizes_and_refusals():
    assert tseq.tconv_q8_codes_bytes(3, 49) == 3 * 56 and tseq.tconv_q8_scales_bytes(3, 49) == 3 * 2
    assert tseq.tconv_q8_codes_bytes(1, 1) == 8 and tseq.tconv_q8_scales_bytes(1, 1) == 1
    assert tseq.tconv_q8_codes_bytes(0, 4) == 0 and tseq.tconv_q8_scales_bytes(4, -1) == 0
    assert tseq.tconv_q8_codes_bytes(1 << 30, 1 << 30) == 0
    lib = tconv._lib
    for rows, inner, dt, want in ((0, 4, 0, -1), (4, 0, 0, -1), (4, 4, 7, -1), (1 << 30, 1 << 30, 0, -7)):
        assert lib.tconv_q8_store(rows, inner, dt, P(0x1000), P(0x2000), P(0x3000), P(0)) == want
        assert lib.tconv_q8_restore(rows, inner, dt, P(0x1000), P(0x2000), P(0x3000), P(0)) == want
    assert lib.tconv_q8_store(4, 4, 0, P(0), P(0x2000), P(0x3000), P(0)) == -1
    assert lib.tconv_q8_store(4, 4, 0, P(0x1004), P(0x2000), P(0x3000), P(0)) == -3
    assert lib.tconv_q8_restore(4, 4, 0, P(0x1000), P(0x2008), P(0x3000), P(0)) == -3


def test_scan_refusals():
    ok = tseq.scan_desc(2, 3, 500, "bf16")
    assert tseq.tconv_scan_states_bytes(ok) > 0
    for bad in (tseq.scan_desc(0, 3, 5), tseq.scan_desc(2, 0, 5), tseq.scan_desc(2, 3, 0), tseq.scan_desc(2, 3, 5, x_row=-1),
                tseq.scan_desc(2, 3, 5, grad_batch=-1)):
        assert _scan(bad) == -1 and _scan_bwd(bad) == -1 and tseq.tconv_scan_states_bytes(bad) == 0
    wrong = tseq.scan_desc(2, 3, 5)
    wrong.dtype = 5
    assert _scan(wrong) == -1
    assert _scan(tseq.scan_desc(1 << 20, 1 << 20, 4)) == -7
    for name in ("x", "gate", "y", "h_last"):
        assert _scan(ok, **{name: 0}) == -1, name
    assert _scan(ok, xc=0x100) == -1                                   # some of the four 8-bit buffers
    assert _scan(ok, xc=0x100, xs=0x200, gc=0x300, gs=0x400, states=0) == -1
    assert _scan(ok, h0=0x4000) == -1                                  # h_last is h0 and L > 1
    assert _scan(ok, x=0x1001) == -3 and _scan(ok, y=0x3002) == -3
    for name in ("x", "gate", "states", "gy", "gx", "gg"):
        assert _scan_bwd(ok, **{name: 0}) == -1, name
    assert _scan_bwd(tseq.scan_desc(2, 3, 500, grad_batch=1499)) == -1   # batch entries of the gradients would overlap
    assert _scan_bwd(ok, gy=0x6002) == -3 and _scan_bwd(ok, gx=0x7001) == -3
    assert tconv._lib.tconv_scan_forward(None, *([P(0x1000)] * 12), 0, P(0)) == -1


def test_norm_refusals():
    lib, ok = tconv._lib, tseq.norm_desc(2, 8, 5)

    def fwd(d, **kw):
        a = dict(x=0x1000, r=0, w=0x2000, sum=0, y=0x3000, rstd=0, yc=0, ys=0, sc=0, ss=0)
        a.update(kw)
        return lib.tconv_norm_forward(ctypes.byref(d), *(P(v) for v in a.values()), P(0))

    def bwd(d, **kw):
        a = dict(s=0x1000, sc=0, ss=0, rstd=0x2000, w=0x3000, gy=0x4000, gs=0, gx=0x5000, gw=0, ws=0)
        a.update(kw)
        return lib.tconv_norm_backward(ctypes.byref(d), *(P(v) for v in a.values()), 0, P(0))

    for bad in (tseq.norm_desc(0, 8, 5), tseq.norm_desc(2, 0, 5), tseq.norm_desc(2, 8, 0), tseq.norm_desc(2, 8, 5, eps=-1.0),
                tseq.norm_desc(2, 8, 5, eps=float("nan"))):
        assert fwd(bad) == -1 and bwd(bad) == -1 and tseq.tconv_norm_workspace_bytes(bad) == 0
    assert fwd(tseq.norm_desc(1 << 30, 1 << 30, 5)) == -7
    assert fwd(tseq.norm_desc((1 << 30) + 1, 1, 33)) == -7             # more blocks of 32 positions than a launch counts
    assert fwd(ok, x=0) == -1 and fwd(ok, w=0) == -1 and fwd(ok, y=0) == -1
    assert fwd(ok, yc=0x100) == -1 and fwd(ok, ss=0x100) == -1
    assert fwd(ok, r=0x100) == -1 and fwd(ok, sum=0x100) == -1          # a residual and its sum go together
    assert fwd(ok, x=0x1008) == -3 and fwd(ok, y=0x3004) == -3
    for name in ("s", "rstd", "w", "gy", "gx"):
        assert bwd(ok, **{name: 0}) == -1, name
    assert bwd(ok, sc=0x100, ss=0x200) == -1                            # the stream and its 8-bit form
    assert bwd(ok, gy=0x4004) == -3


def test_python_refusals():
    x, w = torch.zeros(2, 4, 8), torch.ones(4)
    for call in (lambda: tnn.q8_store(x), lambda: tnn.gated_scan(x, x), lambda: tnn.rms_norm(x, w),
                 lambda: tnn.gated_scan_step(torch.zeros(2, 4), torch.zeros(2, 4), torch.zeros(2, 4))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="checkpoint"):
        tnn.gated_scan(x, x, checkpoint="int4")
    with pytest.raises(ValueError, match="output"):
        tnn.rms_norm(x, w, output="int8")
    with pytest.raises(ValueError, match="checkpoint"):
        tnn.RMSNorm(4, checkpoint=8)
    with pytest.raises(ValueError, match="dtype"):
        tnn.Q8(x, x, (1,), torch.float64).restore()
