"""maxsim_rope and maxsim_clip_grad_norm against their definitions in 64 bits."""
import math
import os
import sys

import pytest
import torch

from paper_2605_29517_amd import autograd as A
from paper_2605_29517_amd import binding as M

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import attention_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def freqs_of(rot, base=10000.0):
    return base ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float32) / rot)


def rope_check(X, freqs, at, got, interleaved, inverse, scale):
    """The rotation in fp32 with a cosine and a sine that are right to about 2^-22, then one rounding: a pair's error is that part of its
    length, and half a unit of the entry."""
    want = R.rope(X, freqs, at, interleaved, inverse, scale)
    rot = 2 * freqs.shape[0]
    x = X.double().abs()
    size = x.clone()
    if interleaved:
        pair = x[..., 0:rot:2] + x[..., 1:rot:2]
        size[..., 0:rot:2] = size[..., 1:rot:2] = pair
    else:
        pair = x[..., :rot // 2] + x[..., rot // 2:rot]
        size[..., :rot // 2] = size[..., rot // 2:rot] = pair
    R.check("rope", got, (want, 2.0 ** -20 * size * abs(scale) + R.UNIT[X.dtype] * want.abs() + R.TINY[X.dtype]))
    assert torch.equal(got[..., rot:], X[..., rot:])


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,d,rot", [(1, 64, 64), (12, 64, 32), (5, 128, 128), (3, 80, 42), (2, 96, 2), (4, 6, 4), (40, 128, 64), (7, 20, 10)])
def test_rope(heads, d, rot, dtype, interleaved, inverse):
    print(heads, d, rot, dtype, interleaved, inverse, flush=True)
    lens = [1, 0, 33, 300, 0, 5, 64]
    off = R.offsets(lens, DEV)
    X = torch.randn(sum(lens), heads, d, generator=gen(1), device=DEV).to(TYPES[dtype])
    at = torch.cat([torch.arange(n) for n in lens]).to(DEV)
    got = M.maxsim_rope(X, freqs_of(rot), offsets=off, interleaved=interleaved, inverse=inverse, scale=1.1)
    torch.cuda.synchronize()
    rope_check(X, freqs_of(rot), at, got, interleaved, inverse, 1.1)
    again = X.clone()
    assert M.maxsim_rope(again, freqs_of(rot), offsets=off, interleaved=interleaved, inverse=inverse, scale=1.1, out=again) is again
    torch.cuda.synchronize()
    assert torch.equal(again, got) or (again.double() - got.double()).abs().max() <= 2.0 ** -20 * X.abs().max() * 4 + 2 * R.UNIT[X.dtype] * X.abs().max()


@pytest.mark.parametrize("tokens", [1, 2, 63, 2500, 70000])
def test_rope_positions(tokens):
    """Given positions, far out and negative ones among them; and rows as positions."""
    X = torch.randn(tokens, 2, 32, generator=gen(2), device=DEV)
    at = torch.randint(-1000, 1 << 20, (tokens,), generator=gen(3), device=DEV, dtype=torch.int32)
    rope_check(X, freqs_of(32), at, M.maxsim_rope(X, freqs_of(32), positions=at), False, False, 1.0)
    rope_check(X, freqs_of(32), torch.arange(tokens, device=DEV), M.maxsim_rope(X, freqs_of(32)), False, False, 1.0)


def test_rope_views():
    """Queries and keys of one projection in one call; rows that are not multiples of 16 bytes; into a view."""
    T, d = 77, 64
    fused = torch.randn(T, 8, d, generator=gen(4), device=DEV).bfloat16()
    at = torch.arange(T, device=DEV)
    part = fused[:, :6]
    want = M.maxsim_rope(part.contiguous(), freqs_of(d))
    assert torch.equal(M.maxsim_rope(part, freqs_of(d)), want)
    M.maxsim_rope(part, freqs_of(d), out=part)
    assert torch.equal(fused[:, :6], want)
    odd = torch.randn(T * 3 * 65 + 1, generator=gen(5), device=DEV).half()[1:].view(T, 3, 65)[:, :, :64]
    for interleaved in (False, True):
        rope_check(odd, freqs_of(d), at, M.maxsim_rope(odd, freqs_of(d), interleaved=interleaved), interleaved, False, 1.0)
    heads_first = torch.randn(4, T, d, generator=gen(6), device=DEV).transpose(0, 1)
    rope_check(heads_first, freqs_of(d), at, M.maxsim_rope(heads_first, freqs_of(d)), False, False, 1.0)


def test_rope_gradient():
    X = torch.randn(50, 3, 32, generator=gen(7), device=DEV).requires_grad_()
    G = torch.randn(50, 3, 32, generator=gen(8), device=DEV)
    off = R.offsets([20, 30], DEV)
    Y = A.rope(X, freqs_of(16), offsets=off, interleaved=True, scale=1.3)
    (Y * G).sum().backward()
    at = torch.cat((torch.arange(20), torch.arange(30))).to(DEV)
    rope_check(G, freqs_of(16), at, torch.cat((X.grad[..., :16], G[..., 16:]), -1), True, True, 1.3)
    assert torch.equal(X.grad[..., 16:], G[..., 16:])
    # a linear map: its difference along any direction is the gradient's product with it
    step = torch.randn(50, 3, 32, generator=gen(9), device=DEV)
    along = ((M.maxsim_rope((X + step).detach(), freqs_of(16), offsets=off, interleaved=True, scale=1.3).double() - Y.detach().double()) * G.double()).sum()
    assert abs(along - (X.grad.double() * step.double()).sum()) < 1e-4 * (X.grad.double() * step.double()).norm() + 1e-4
    grad = A.rope(torch.ones(4, 2, 8, device=DEV, requires_grad=True), freqs_of(8)).sum()  # an expanded view comes back
    grad.backward()


def test_rope_refusals():
    X = torch.zeros(4, 2, 8, device=DEV)
    with pytest.raises(M.MaxSimError, match="rot"):
        M.maxsim_rope(X, freqs_of(16))
    with pytest.raises(M.MaxSimError, match="dtype"):
        M.maxsim_rope(X, freqs_of(8).double())
    with pytest.raises(M.MaxSimError, match="dtype"):
        M.maxsim_rope(X.double(), freqs_of(8))
    with pytest.raises(M.MaxSimError, match="positions"):
        M.maxsim_rope(X, freqs_of(8), positions=torch.zeros(5, dtype=torch.int32, device=DEV))
    with pytest.raises(M.MaxSimError, match="GPU"):
        M.maxsim_rope(X.cpu(), freqs_of(8))
    with pytest.raises(M.MaxSimError, match="invalid"):
        M.maxsim_rope(X, freqs_of(8), out=X[:, :1].expand(-1, 2, -1))


def clip_check(grads, max_norm, out, norm):
    total = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    # the norm is rounded to fp32 once, the factor takes a sum, a quotient and a product more
    assert abs(float(norm) - total) <= 2.0 ** -23 * total
    by = min(1.0, max_norm / (total + 1e-6))
    for g, o in zip(grads, out):
        want = g.double() * by
        R.check("clipped", o, (want, (R.UNIT[g.dtype] + 2.0 ** -21) * want.abs() + R.TINY[g.dtype]))


@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e9])
@pytest.mark.parametrize("sizes", [[1], [4096], [4095, 4097, 1, 0, 8192], [0, 0, 3, 0], [3] * 109, [5] * 110, [7] * 111, [1000, 0, 33] * 120, [5_000_011, 12]])
def test_clip(sizes, max_norm):
    print(len(sizes), max_norm, flush=True)
    kinds = list(TYPES.values())
    grads = [(torch.randn(n, generator=gen(i), device=DEV) * 0.1).to(kinds[i % 3]) for i, n in enumerate(sizes)]
    out = [torch.full_like(g, float("nan")) for g in grads]
    norm = M.maxsim_clip_grad_norm(grads, max_norm, out=out)
    clip_check(grads, max_norm, out, norm)
    inplace = [g.clone() for g in grads]
    norm2 = M.maxsim_clip_grad_norm(inplace, max_norm)
    assert torch.equal(norm, norm2) and all(torch.equal(a, b) for a, b in zip(inplace, out))


def test_clip_views_and_extremes():
    flat = torch.randn(30_003, generator=gen(1), device=DEV).half()
    grads = [flat[1:10_000], flat[10_001:20_002], flat[20_003:]]  # not multiples of 16 bytes
    out = torch.full_like(flat, 7.0)
    outs = [out[1:10_000], out[10_001:20_002], out[20_003:]]
    clip_check(grads, 1.0, outs, M.maxsim_clip_grad_norm(grads, 1.0, out=outs))
    assert float(out[0]) == float(out[10_000]) == float(out[20_002]) == 7.0
    huge = [torch.full((5000,), 1e30, device=DEV), torch.full((10,), 1e-30, device=DEV)]  # squares beyond fp32
    norm = M.maxsim_clip_grad_norm(huge, 1.0)
    assert abs(float(norm) / (1e30 * math.sqrt(5000)) - 1) < 1e-6
    assert torch.allclose(huge[0], torch.full_like(huge[0], 1 / math.sqrt(5000)), rtol=1e-6)
    bad = torch.ones(5000, device=DEV)
    for value in (float("inf"), float("nan")):
        bad[4999] = value
        fine = torch.ones(3, device=DEV)
        norm = M.maxsim_clip_grad_norm([fine, bad.clone()], 1.0)
        assert not math.isfinite(float(norm))
        assert (fine == 0).all() if value == float("inf") else fine.isnan().all()


def test_clip_on_another_stream_and_in_a_graph():
    M.maxsim_init()
    grads = [torch.randn(n, generator=gen(n), device=DEV) for n in (100_000, 33)]
    out = [torch.empty_like(g) for g in grads]
    ws = torch.empty(M.load().maxsim_clip_workspace(2), dtype=torch.uint8, device=DEV)
    norm = torch.empty(1, device=DEV)
    M.maxsim_clip_grad_norm(grads, 1.0, out=out, norm=norm, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.maxsim_clip_grad_norm(grads, 1.0, out=out, norm=norm, workspace=ws)
    for k in range(3):
        grads[0].mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        clip_check(grads, 1.0, out, norm)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        twice = [g * 2 for g in grads]
        norm = M.maxsim_clip_grad_norm(twice, 1.0)
    side.synchronize()
    clip_check([g * 2 for g in grads], 1.0, twice, norm)


def test_clip_refusals():
    g = torch.ones(4, device=DEV)
    with pytest.raises(M.MaxSimError, match="tensor"):
        M.maxsim_clip_grad_norm([], 1.0)
    with pytest.raises(M.MaxSimError, match="dtype"):
        M.maxsim_clip_grad_norm([g.double()], 1.0)
    with pytest.raises(M.MaxSimError, match="contiguous"):
        M.maxsim_clip_grad_norm([torch.ones(4, 4, device=DEV).t()[:2]], 1.0)
    with pytest.raises(M.MaxSimError, match="shape"):
        M.maxsim_clip_grad_norm([g], 1.0, out=[torch.ones(5, device=DEV)])
    for bad in (-1.0, float("nan")):
        with pytest.raises(M.MaxSimError, match="invalid"):
            M.maxsim_clip_grad_norm([g], bad)
    with pytest.raises(M.MaxSimError, match="scratch|workspace"):
        M.maxsim_clip_grad_norm([g], 1.0, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
