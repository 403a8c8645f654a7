"""The entry points of rotary positions, attention and clipping without a GPU: refusals, workspaces, and what the compiler makes of the
parts that are assembly."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2605_29517_amd import binding as M
from paper_2605_29517_amd import build as B

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
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


def test_rope_refusals(L, p):
    good = [p, 4, 2, 8, 16, 8, 1, p, 8, None, None, 0, 1.0, 0, 0, p, 16, 8, None]

    def call(**changed):
        names = ("X tokens heads d xt xh dtype freqs rot positions offsets b scale neighbours inverse Y yt yh stream").split()
        return L.maxsim_rope(*[changed.get(n, g) for n, g in zip(names, good)])

    odd = ctypes.c_void_p(p.value + 1)
    for bad in (dict(X=None), dict(Y=None), dict(freqs=None), dict(tokens=0), dict(heads=0), dict(rot=0), dict(rot=3), dict(rot=10), dict(dtype=3), dict(X=odd), dict(xt=-1),
                dict(yt=4), dict(yh=0), dict(offsets=p, b=0), dict(scale=float("nan"))):
        assert call(**bad) == INVALID, bad
    assert call(d=5000, rot=5000, yt=10000, yh=5000) == UNSUPPORTED
    assert call(tokens=1 << 31) == UNSUPPORTED


def attention(L, p, backward=False, **changed):
    names = ("Q K V strides qo ko b tq tk hq hkv d dtype causal scale O lse ws bytes stream").split()
    good = dict(zip(names, [p, p, p, None, p, p, 2, 100, 100, 4, 2, 64, 1, 1, 0.125, p, p, p, 1 << 40, None]))
    good.update(dO=p, dQ=p, dK=p, dV=p)
    good.update(changed)
    if backward:
        names = ("Q K V O lse dO strides qo ko b tq tk hq hkv d dtype causal scale dQ dK dV ws bytes stream").split()
    return (L.maxsim_attention_backward if backward else L.maxsim_attention)(*[good[n] for n in names])


@pytest.mark.parametrize("backward", [False, True])
def test_attention_refusals(L, p, backward):
    odd = ctypes.c_void_p(p.value + 8)
    for bad in (dict(Q=None), dict(V=None), dict(O=None), dict(qo=None), dict(ko=None), dict(b=0), dict(tq=0), dict(tk=0), dict(hq=0), dict(hkv=3), dict(dtype=5), dict(scale=0.0),
                dict(scale=float("inf")), dict(scale=float("nan")), dict(K=odd)):
        assert attention(L, p, backward, **bad) == INVALID, bad
    for bad in (dict(dtype=0), dict(d=12), dict(d=264), dict(tq=1 << 30), dict(tk=1 << 30), dict(b=1 << 24)):
        assert attention(L, p, backward, **bad) == UNSUPPORTED, bad
    n = 16 if backward else 8
    plain = [256, 64, 128, 64, 128, 64, 256, 64, 256, 64, 256, 64, 128, 64, 128, 64][:n]
    for i, value in ((0, 252), (1, 60), (2, -8), (7, 0) if not backward else (11, 0), (6, 8) if not backward else (12, 8)):
        strides = list(plain)
        strides[i] = value
        assert attention(L, p, backward, strides=(ctypes.c_int64 * n)(*strides)) == INVALID, (i, value)
    strides = [1 << 24] + plain[1:]
    assert attention(L, p, backward, strides=(ctypes.c_int64 * n)(*strides)) == UNSUPPORTED
    if backward:
        for bad in (dict(lse=None), dict(dO=None), dict(dQ=None), dict(dK=None), dict(dV=None), dict(ws=None)):
            assert attention(L, p, True, **bad) == INVALID, bad
        assert attention(L, p, True, bytes=100 * 4 * 8 - 1) == SCRATCH


def test_workspaces(L):
    """None for a long prompt; for a single token after many keys, its pieces' results; for the gradient, two numbers a row at least."""
    assert L.maxsim_attention_workspace(1, 8192, 8192, 32, 8, 128) == 0
    assert L.maxsim_attention_workspace(64, 2048, 2048, 12, 12, 64) == 0
    one = L.maxsim_attention_workspace(1, 1, 100_003, 16, 2, 128)
    assert one % (16 * 129 * 4) == 0 and 64 <= one // (16 * 129 * 4) <= 256
    assert attention_scratch(L, one)
    assert L.maxsim_attention_backward_workspace(4, 16384, 16384, 32, 8, 128) == 16384 * 32 * 8
    assert L.maxsim_attention_backward_workspace(1, 1000, 1000, 8, 1, 128) > 1000 * 8 * 8
    assert L.maxsim_attention_workspace(0, 1, 1, 1, 1, 64) == L.maxsim_attention_backward_workspace(1, 1, 1, 1, 1, 300) == 0
    assert L.maxsim_clip_workspace(0) == 0 and L.maxsim_clip_workspace(1000) > L.maxsim_clip_workspace(10) > 0


def attention_scratch(L, needed):
    keep = (ctypes.c_char * 4096)()
    at = ctypes.c_void_p((ctypes.addressof(keep) + 255) & ~255)
    return attention(L, at, b=1, tq=1, tk=100_003, hq=16, hkv=2, d=128, bytes=needed - 1) == SCRATCH


def test_clip_refusals(L, p):
    def call(n=1, max_norm=1.0, numel=4, dtype=0, g=p, out=p, norm=p, ws=p, size=1 << 30):
        P = ctypes.c_void_p * 1
        return L.maxsim_clip_grad_norm(P(g), P(out), (ctypes.c_int64 * 1)(numel), (ctypes.c_int32 * 1)(dtype), n, max_norm, norm, ws, size, None)

    odd = ctypes.c_void_p(p.value + 2)
    for bad in (dict(n=0), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(numel=-1), dict(dtype=3), dict(g=None), dict(out=None), dict(norm=None), dict(ws=None), dict(g=odd)):
        assert call(**bad) == INVALID, bad
    assert call(size=16) == SCRATCH
    assert call(numel=1 << 51) == UNSUPPORTED


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
@pytest.mark.parametrize("source", ["attention.hip", "attention_backward.hip"])
def test_copies_to_lds(tmp_path, source):
    """The copies are assembly that sets m0 itself: nothing else may use it, each copy has its own setting and the cycle between, and apart
    from the wait at a tile's arrival no loop waits for loads (the compiler must not have a load of its own in flight there)."""
    out = tmp_path / "kernels.s"
    subprocess.run([HIPCC] + B.FLAGS + ["--cuda-device-only", "-S", os.path.join(B.CSRC, source), "-o", str(out)], check=True, stderr=subprocess.DEVNULL)
    kernels = re.findall(r"^(_ZN\S*attn_(?:fwd|few|dq|dkv)_kernel\S*):(.*?)\.Lfunc_end", out.read_text(), re.S | re.M)
    assert len(kernels) >= 10
    for name, body in kernels:
        lines = [x for x in (line.split(";")[0].strip() for line in body.split("\n")) if x and not x.startswith(".p2") and not x.startswith("#")]
        copies = 0
        for i, line in enumerate(lines):
            if "m0" in re.findall(r"\w+", line):
                assert line.startswith("s_mov_b32 m0,") and lines[i + 1] == "s_nop 0" and lines[i + 2].startswith("global_load_lds_"), (name, lines[i:i + 3])
            copies += line.startswith("global_load_lds_")
        assert copies and sum(x.startswith("s_mov_b32 m0,") for x in lines) == copies, name
        # the tightest loop around MFMAs: from a label to a branch back to it
        labels = {x[:-1]: i for i, x in enumerate(lines) if x.endswith(":")}
        loops = [lines[labels[x.split()[-1]]:i] for i, x in enumerate(lines) if x.startswith(("s_cbranch", "s_branch")) and labels.get(x.split()[-1], i) < i]
        loop = min((x for x in loops if any("v_mfma" in y for y in x)), key=len)
        assert not [x for x in loop if re.match(r"(global|flat|scratch|buffer)_load_(?!lds)", x)], name
