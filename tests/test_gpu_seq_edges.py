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
        assert torch.isfinite(gx).all() and (gg.abs() < 1e-30).all()
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
