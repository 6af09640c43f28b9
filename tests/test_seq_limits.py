"""Sizes at the ends of what the sequence and storage operators take (no GPU needed)."""
import ctypes

import pytest

from paper_2504_06881_b200 import tconv, tseq

P = ctypes.c_void_p
MOST = 2 ** 31 - 1


def _norm(d):
    """What forward and backward say before anything is launched: x, then grad_x, is misaligned."""
    lib = tconv._lib
    fwd = lib.tconv_norm_forward(ctypes.byref(d), *(P(v) for v in (0x1004, 0, 0x2000, 0, 0x3000, 0, 0, 0, 0, 0)), P(0))
    bwd = lib.tconv_norm_backward(ctypes.byref(d), *(P(v) for v in (0x1000, 0, 0, 0x2000, 0x3000, 0x4000, 0, 0x5004, 0, 0)), 0, P(0))
    return fwd, bwd


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C,P_", [(1, MOST, 1), (1, MOST - 30, 1), (1, MOST - 31, 1), (1, MOST - 4094, 1), (MOST, 1, 1), (MOST - 2, 8, 1),
                                    (MOST - 4094, 1, 1), (1, MOST, 40), (1, MOST - 3, 33), (1, MOST - 4094, 64)])
def test_norm_refuses_counts_that_32_bits_do_not_hold(N, C, P_, dtype):
    """Rounding C up to a multiple of 32, or stepping past the last channel, would leave 32 bits."""
    d = tseq.norm_desc(N, C, P_, dtype)
    assert _norm(d) == (-7, -7) and tseq.tconv_norm_workspace_bytes(d) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,C,P_", [(1, MOST - 4095, 1), (1, MOST - 4096, 1), (MOST - 4095, 1, 1), (MOST - 4097, 8, 1), (1, MOST - 4095, 40),
                                    (1, MOST - 4098, 33), (1, 2 ** 30, 7)])
def test_norm_takes_counts_up_to_there(N, C, P_, dtype):
    """Partial sums of grad_weight: some of C each, as many as blocks or row groups (1216 and 1184 at most)."""
    d = tseq.norm_desc(N, C, P_, dtype)
    assert _norm(d) == (-3, -3)
    parts, rest = divmod(tseq.tconv_norm_workspace_bytes(d), 4 * C)
    assert rest == 0 and 1 <= parts <= 1216
