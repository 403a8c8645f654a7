"""maxsim_norm_rope and maxsim_norm_rope_backward against their definitions in 64 bits."""
import os
import sys

import pytest
import torch

from paper_2605_29517_amd import autograd as A
from paper_2605_29517_amd import binding as M

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import attention_reference as R  # noqa: E402
import training_reference as T  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def freqs_of(rot, base=10000.0):
    return base ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float32) / rot)


def randn(*shape, seed, dtype="f32"):
    return torch.randn(*shape, generator=gen(seed), device=DEV).to(TYPES[dtype])


def both(X, dY, freqs, qw, kw, q_heads, at, how, interleaved=False, scale=1.0, eps=1e-6):
    """Forward and backward against the definitions; returns both results."""
    Y = M.maxsim_norm_rope(X, freqs, qw, kw, q_heads=q_heads, eps=eps, interleaved=interleaved, scale=scale, **how)
    got = M.maxsim_norm_rope_backward(X, dY, freqs, qw, kw, q_heads=q_heads, eps=eps, interleaved=interleaved, scale=scale, **how)
    torch.cuda.synchronize()
    q = X.shape[1] if q_heads is None else q_heads
    R.check("Y", Y, T.norm_rope(X, freqs, qw, kw, q, eps, at, interleaved, scale))
    want = T.norm_rope_backward(X, dY, freqs, qw, kw, q, eps, at, interleaved, scale)
    for name, g, w, there in zip(("dX", "dq_weight", "dk_weight"), got, want, (True, qw is not None, kw is not None)):
        assert (g is not None) == there
        if there:
            R.check(name, g, w)
    return Y, got


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,weights", [("f32", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("hq,hkv,d,rot", [(1, 0, 64, 64), (12, 12, 64, 32), (5, 1, 128, 128), (0, 3, 80, 42), (2, 2, 96, 2), (4, 3, 6, 4), (32, 8, 128, 64), (3, 2, 20, 10), (1, 1, 2, 2), (2, 1, 512, 512),
                                          (2, 3, 256, 256), (1, 2, 511, 510), (7, 5, 48, 48), (6, 2, 80, 40), (3, 1, 84, 42), (2, 1, 504, 24), (1, 1, 500, 500), (1, 1, 510, 510),
                                          (2, 2, 508, 4)])
def test_norm_rope(hq, hkv, d, rot, dtype, weights, interleaved):
    print(hq, hkv, d, rot, dtype, weights, interleaved, flush=True)
    lens = [1, 0, 33, 300, 0, 5, 64]
    n = sum(lens)
    at = torch.cat([torch.arange(k) for k in lens]).to(DEV)
    qw, kw = ((1 + 0.2 * randn(d, seed=s)).to(TYPES[weights]) for s in (1, 2))
    X, dY = randn(n, hq + hkv, d, seed=3, dtype=dtype), randn(n, hq + hkv, d, seed=4, dtype=dtype)
    X[40, 0] = 0  # a row that eps alone keeps apart from zero
    how = dict(offsets=R.offsets(lens, DEV))
    Y, (dX, dqw, dkw) = both(X, dY, freqs_of(rot), qw, kw, hq, at, how, interleaved, scale=1.1)
    again = X.clone()
    assert M.maxsim_norm_rope(again, freqs_of(rot), qw, kw, q_heads=hq, interleaved=interleaved, scale=1.1, out=again, **how) is again
    assert torch.equal(again, Y)
    for into in (X.clone(), dY.clone()):
        x, g = (into, dY) if torch.equal(into, X) else (X, into)
        r = M.maxsim_norm_rope_backward(x, g, freqs_of(rot), qw, kw, q_heads=hq, interleaved=interleaved, scale=1.1, dX=into, **how)
        torch.cuda.synchronize()
        assert r[0] is into and torch.equal(into, dX) and torch.equal(r[1], dqw) and torch.equal(r[2], dkw)


@pytest.mark.parametrize("tokens", [1, 2, 63, 2500, 70_000])
def test_positions(tokens):
    """Given positions, far out and negative ones among them; and rows as positions; one kind of heads, with and without weights."""
    X, dY = randn(tokens, 2, 32, seed=5), randn(tokens, 2, 32, seed=6)
    at = torch.randint(-1000, 1 << 20, (tokens,), generator=gen(7), device=DEV, dtype=torch.int32)
    both(X, dY, freqs_of(32), 1 + 0.1 * randn(32, seed=8), None, None, at, dict(positions=at))
    both(X, dY, freqs_of(16), None, 1 + 0.1 * randn(32, seed=8), 1, torch.arange(tokens, device=DEV), dict())
    both(X, dY, freqs_of(16), None, None, None, torch.arange(tokens, device=DEV), dict(), eps=0.5)


def test_weights_without_heads():
    X, w = randn(5, 2, 8, seed=9), torch.ones(8, device=DEV)
    _, (_, dq, dk) = both(X, X, freqs_of(8), w, w, 2, torch.arange(5, device=DEV), dict())
    assert (dk == 0).all() and (dq != 0).any()


def test_views():
    """Queries and keys of one fused projection and into a gradient of the whole of it; rows that are not multiples of 16 bytes; heads before tokens."""
    n, d, w = 77, 64, 1 + 0.1 * randn(64, seed=10)
    at = torch.arange(n, device=DEV)
    for dtype in TYPES:
        fused, grads = randn(n, 8, d, seed=11, dtype=dtype), randn(n, 6, d, seed=12, dtype=dtype)
        Y, (dX, dq, dk) = both(fused[:, :6], grads, freqs_of(d), w, w, 4, at, dict())
        whole = torch.full_like(fused, 7.0)
        M.maxsim_norm_rope_backward(fused[:, :6], grads, freqs_of(d), w, w, q_heads=4, dX=whole[:, :6])
        assert torch.equal(whole[:, :6], dX) and (whole[:, 6:] == 7).all()
        M.maxsim_norm_rope(fused[:, :6], freqs_of(d), w, w, q_heads=4, out=fused[:, :6])
        assert torch.equal(fused[:, :6], Y)
        odd = randn(n * 3 * 65 + 1, seed=13, dtype=dtype)[1:].view(n, 3, 65)[:, :, :64]
        for interleaved in (False, True):
            both(odd, odd.contiguous(), freqs_of(d), w, None, None, at, dict(), interleaved)
        turned = randn(3, n, d, seed=14, dtype=dtype).transpose(0, 1)
        both(turned, turned.contiguous(), freqs_of(32), w, w, 1, at, dict())


def test_many_rows_of_one_head():
    """More rows than the gradient's workgroups take at a time, and one row alone."""
    for n, h in ((100_000, 1), (1, 1), (3, 200)):
        X, dY = randn(n, h, 16, seed=15, dtype="bf16"), randn(n, h, 16, seed=16, dtype="bf16")
        both(X, dY, freqs_of(16), 1 + 0.1 * randn(16, seed=17), None, None, torch.arange(n, device=DEV), dict())


def test_large_and_small_entries():
    """fp16 at the ends of its range, fp32 far beyond it: squares are fp32."""
    for dtype, by in (("f16", 6e4), ("f16", 1e-4), ("f32", 1e17), ("f32", 1e-15), ("bf16", 1e16)):
        X = (randn(9, 2, 64, seed=18).clamp(-1, 1) * by).to(TYPES[dtype])
        Y = M.maxsim_norm_rope(X, freqs_of(64), eps=1e-12)
        R.check(dtype, Y, T.norm_rope(X, freqs_of(64), None, None, 2, 1e-12, torch.arange(9, device=DEV), False, 1.0))


def test_differentiable():
    n, d = 40, 24
    X = randn(n, 5, d, seed=19).requires_grad_()
    qw, kw = ((1 + 0.1 * randn(d, seed=s)).requires_grad_() for s in (20, 21))
    off, G = R.offsets([10, 30], DEV), randn(n, 5, d, seed=22)
    at = torch.cat((torch.arange(10), torch.arange(30))).to(DEV)
    f = lambda x, q, k: M.maxsim_norm_rope(x.contiguous(), freqs_of(16), q, k, q_heads=3, offsets=off, interleaved=True, scale=1.3)  # noqa: E731
    Y = A.norm_rope(X, freqs_of(16), qw, kw, q_heads=3, offsets=off, interleaved=True, scale=1.3)
    (Y * G).sum().backward()
    want = T.norm_rope_backward(X.detach(), G, freqs_of(16), qw.detach(), kw.detach(), 3, 1e-6, at, True, 1.3)
    for t, w in zip((X, qw, kw), want):
        R.check("gradient", t.grad, w)
    # against differences of the kernel's own results along a direction: the curvature leaves h^2 of the third derivative, the roundings 2^-22 / h of the values
    h = 2.0 ** -7
    steps = [randn(*t.shape, seed=23 + i) for i, t in enumerate((X, qw, kw))]
    ends = [f(*((t.detach() + s * h * v) for t, v in zip((X, qw, kw), steps))).double() for s in (1, -1)]
    along = ((ends[0] - ends[1]) * G.double()).sum() / (2 * h)
    exact = sum((t.grad.double() * v.double()).sum() for t, v in zip((X, qw, kw), steps))
    assert abs(along - exact) < 2e-3 * sum((t.grad.double() * v.double()).norm() for t, v in zip((X, qw, kw), steps)) + n * 5 * d * 2.0 ** -22 / h
    # 16-bit activations, weights in fp32; a transposed view and an expanded gradient
    x = randn(5, n, d, seed=26, dtype="bf16").transpose(0, 1).requires_grad_()
    A.norm_rope(x, freqs_of(16), qw, kw, q_heads=3, offsets=off).float().sum().backward()
    assert x.grad.dtype == torch.bfloat16 and qw.grad.dtype == torch.float32
    A.norm_rope(X, freqs_of(16), None, None).sum().backward()


def test_graph_and_streams():
    M.maxsim_init()
    n, d = 500, 64
    X, dY, w = randn(n, 6, d, seed=27, dtype="bf16"), randn(n, 6, d, seed=28, dtype="bf16"), torch.ones(d, device=DEV)
    ws = torch.empty(M.load().maxsim_norm_rope_backward_workspace(n, 6, d), dtype=torch.uint8, device=DEV)
    Y, dX = torch.empty_like(X), torch.empty_like(X)

    def step():
        M.maxsim_norm_rope(X, freqs, w, w, q_heads=4, out=Y)
        return M.maxsim_norm_rope_backward(X, dY, freqs, w, w, q_heads=4, dX=dX, workspace=ws)

    freqs = freqs_of(d)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        X.copy_(randn(n, 6, d, seed=30 + k, dtype="bf16"))
        w.copy_(1 + 0.1 * randn(d, seed=40 + k))
        graph.replay()
        torch.cuda.synchronize()
        kept = [Y.clone()] + [t.clone() for t in got]
        both(X, dY, freqs, w, w, 4, torch.arange(n, device=DEV), dict())
        eager = [M.maxsim_norm_rope(X, freqs, w, w, q_heads=4), *M.maxsim_norm_rope_backward(X, dY, freqs, w, w, q_heads=4)]
        assert all(torch.equal(a, b) for a, b in zip(kept, eager))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        twice = dY * 2
        r = M.maxsim_norm_rope_backward(X, twice, freqs, w, w, q_heads=4)
    side.synchronize()
    assert torch.equal(r[1], eager[2] * 2) and torch.equal(r[2], eager[3] * 2)


def test_refusals():
    X, w, f = torch.zeros(4, 2, 8, device=DEV), torch.ones(8, device=DEV), freqs_of(8)
    for call, match in ((lambda: M.maxsim_norm_rope(X, freqs_of(16)), "rot"), (lambda: M.maxsim_norm_rope(X, f, w, w), "q_heads"), (lambda: M.maxsim_norm_rope(X, f, w, w, q_heads=3), "q_heads"),
                        (lambda: M.maxsim_norm_rope(X, f, w[:4]), "shape"), (lambda: M.maxsim_norm_rope(X, f, w, w.half(), q_heads=1), "share"), (lambda: M.maxsim_norm_rope(X, f, w.double()), "dtype"),
                        (lambda: M.maxsim_norm_rope(X.double(), f), "dtype"), (lambda: M.maxsim_norm_rope(X.cpu(), f), "GPU"), (lambda: M.maxsim_norm_rope(X, f, eps=-1.0), "invalid"),
                        (lambda: M.maxsim_norm_rope(X, f, eps=float("nan")), "invalid"), (lambda: M.maxsim_norm_rope(X, f, out=X[:, :1].expand(-1, 2, -1)), "invalid"),
                        (lambda: M.maxsim_norm_rope(X, f, positions=torch.zeros(5, dtype=torch.int32, device=DEV)), "positions"),
                        (lambda: M.maxsim_norm_rope(torch.zeros(2, 1, 514, device=DEV), f), "width|size"),
                        (lambda: M.maxsim_norm_rope_backward(X, X.half(), f), "dtype"), (lambda: M.maxsim_norm_rope_backward(X, X[:3], f), "shape"),
                        (lambda: M.maxsim_norm_rope_backward(X, X, f, w, workspace=torch.empty(16, dtype=torch.uint8, device=DEV)), "scratch|workspace")):
        with pytest.raises(M.MaxSimError, match=match):
            call()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,by,eps", [(512, 8e17, 1e-6), (340, 1e18, 1e-6), (64, 2.3e18, 1e-6), (512, 1e-18, 0.0), (64, 1e-18, 0.0), (2, 1.3e19, 0.0)])
def test_the_ends_of_what_squares_can_hold(d, by, eps, interleaved):
    """Rows whose squares add up to just less than fp32 holds, and to as little as it holds with all of its digits."""
    sign = randn(6, 3, d, seed=51).sign()
    X, dY = sign * by, randn(6, 3, d, seed=52)
    X[1] *= 0.5 + 0.5 * torch.rand(3, d, generator=gen(53), device=DEV)
    w = 1 + 0.1 * randn(d, seed=54)
    assert d * by * by * (1 + d * 2.0 ** -24) < torch.finfo(torch.float32).max and (eps > 0 or 0.25 * by * by > 2.0 ** -126)
    both(X, dY, freqs_of(d // 2 * 2), w, w, 2, torch.arange(6, device=DEV), dict(), interleaved, eps=eps)
