"""Outputs whose rows would lie over one another are refused before anything is launched (no GPU needed); layouts whose rows lie apart are not."""
import ctypes

import pytest

from paper_2605_29517_amd import binding as M

INVALID, UNSUPPORTED, SCRATCH = -1, -2, -4


@pytest.fixture(scope="module")
def L():
    return M.load()


@pytest.fixture(scope="module")
def p():
    keep = (ctypes.c_char * 4096)()
    at = ctypes.c_void_p((ctypes.addressof(keep) + 255) & ~255)
    at.keep = keep
    return at


# strides of token and head of an output [100, 4, 64]
APART = [(256, 64), (512, 64), (64, 6400), (72, 7200), (256, 64 * 1000), (1 << 20, 64)]
OVER_ONE_ANOTHER = [(64, 64), (64, 128), (192, 64), (128, 64), (64, 640), (72, 72), (248, 64)]


@pytest.mark.parametrize("strides", APART + OVER_ONE_ANOTHER)
def test_rotary_positions(L, p, strides):
    """(Heads 150 times as wide, which are wider than rotary positions go, end the call where the strides do not.)"""
    rc = L.maxsim_rope(p, 100, 4, 9600, 4 * 9600, 9600, 1, p, 9600, None, None, 0, 1.0, 0, 0, p, 150 * strides[0], 150 * strides[1], None)
    assert rc == (INVALID if strides in OVER_ONE_ANOTHER else UNSUPPORTED)


@pytest.mark.parametrize("strides", APART + OVER_ONE_ANOTHER)
@pytest.mark.parametrize("which", range(4))
def test_attention(L, p, which, strides):
    """(A workspace that is too small ends the call where the strides do not: the key side of the gradient is split for these sizes.)"""
    plain = [256, 64] * 8
    hq = hkv = 4
    if which == 0:
        args = (ctypes.c_int64 * 8)(*(plain[:6] + list(strides)))
        need = L.maxsim_attention_workspace(1, 100, 20000, hq, hkv, 64)
        assert need > 0
        rc = L.maxsim_attention(p, p, p, args, p, p, 1, 100, 20000, hq, hkv, 64, 1, 1, 0.125, p, p, p, need - 1, None)
    else:
        full = list(plain)
        full[8 + 2 * which:10 + 2 * which] = strides
        rc = L.maxsim_attention_backward(p, p, p, p, p, p, (ctypes.c_int64 * 16)(*full), p, p, 1, 100, 100, hq, hkv, 64, 1, 1, 0.125, p, p, p, p, 16, None)
    assert rc == (INVALID if strides in OVER_ONE_ANOTHER else SCRATCH)
