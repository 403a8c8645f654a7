"""The range of the softmax's scale (no GPU needed)."""
import ctypes

import pytest

from paper_2605_29517_amd import binding as M

INVALID, SCRATCH = -1, -4


@pytest.mark.parametrize("scale,code", [(0.99e-30, INVALID), (1e-38, INVALID), (1e-45, INVALID), (1.01e-30, SCRATCH), (0.99e30, SCRATCH), (1.01e30, INVALID), (-1.0, INVALID)])
def test_scales(scale, code):
    """The gradient starts its sums at -lse / scale, which has to be a finite number. (A workspace that is too small ends the call where the scale does not.)"""
    L = M.load()
    keep = (ctypes.c_char * 4096)()
    p = ctypes.c_void_p((ctypes.addressof(keep) + 255) & ~255)
    assert L.maxsim_attention_backward(p, p, p, p, p, p, None, p, p, 1, 100, 100, 4, 4, 64, 1, 1, scale, p, p, p, p, 16, None) == code
    assert L.maxsim_attention(p, p, p, None, p, p, 1, 100, 20000, 4, 4, 64, 1, 1, scale, p, p, p, 16, None) == code
