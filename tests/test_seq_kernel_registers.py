"""Registers and spills of the sequence operators' kernels that the launch bounds hold down (no GPU needed)."""
import pytest

import nvcc_probe
from paper_2504_06881_b200 import build


def _resources(monkeypatch, header, names):
    monkeypatch.setattr(nvcc_probe, "NVCC", build._nvcc_base(verbose=True, std="c++20"))     # as its unit is compiled
    return nvcc_probe.resources(header, names)


def test_recurrence(monkeypatch):
    """Seven blocks of 128 threads an SM; some 32 bytes of a thread wait in local memory at most."""
    names = [f"scan_{way}_kernel<{t}, {q8}, {acc}, 32, 0>" for way in ("fwd", "bwd") for t in ("float", "__nv_bfloat16")
             for q8 in ("false", "true") for acc in (2, 3)]
    got = _resources(monkeypatch, "tconv_scan.cuh", names)
    assert all(regs <= 65536 // 128 // 7 // 8 * 8 and spilled <= 32 for regs, spilled in got.values()), got


@pytest.mark.parametrize("dtype,vec", [("float", 4), ("__nv_bfloat16", 8)])
def test_norm_backward(monkeypatch, dtype, vec):
    """Sixteen warps an SM: 128 registers.  Without spills but for 32 single values a thread (maps of odd size with 257 to 512
    channels), where the stream kept in 8 bits takes a word a value more than there are registers for."""
    last = (vec, 16, 8 if vec == 4 else 4)
    names = [f"norm_bwd_cols_kernel<{dtype}, {v}, {w}, {r}, {res}, {q8}>" for v, w, r in (last, (1, 8, 16), (1, 16, 16), (1, 16, 32))
             for res in ("false", "true") for q8 in ("false", "true")]
    got = _resources(monkeypatch, "tconv_norm.cuh", names)
    for name, (regs, spilled) in got.items():
        known = 432 if "1, 16, 32" in name and name.endswith("true>") else 32
        assert regs <= 128 and spilled <= known, (name, regs, spilled)
