"""Embedding, norms with rotary positions and distillation of 256 MB and more, whose reads and writes carry the streaming hint: the same bits as from calls for some of the
rows each, which do not, or, where the order of sums differs, against the definitions in 64 bits."""
import os
import sys

import pytest
import torch

from paper_2605_29517_amd import binding as M

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import attention_reference as R  # noqa: E402
import training_reference as T  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HINT = 256 << 20  # bytes read and written


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(*shape, seed, dtype="f32"):
    out = torch.empty(*shape, device=DEV, dtype=TYPES[dtype])
    return out.normal_(generator=gen(seed))


def odd(*shape, seed, dtype, room=3):
    """Rows that begin at any entry and lie `room` entries apart."""
    *outer, d = shape
    return randn(*outer, d + room, seed=seed, dtype=dtype)[..., 1:1 + d]


def parts(n, k):
    at = [n * i // k for i in range(k + 1)]
    return [slice(a, b) for a, b in zip(at, at[1:])]


@pytest.mark.parametrize("dtype,to,n,d", [("f16", "f32", 70_003, 1031), ("f32", "bf16", 70_003, 2050), ("bf16", "bf16", 140_001, 1024), ("f32", "f32", 40_000, 1804)])
def test_embed(dtype, to, n, d):
    print(dtype, to, n, d, flush=True)
    W = randn(3001, d, seed=1, dtype=dtype)
    tokens = torch.randint(-5, 3010, (n,), generator=gen(2), device=DEV, dtype=torch.int32)
    Y = M.maxsim_embed(W, tokens, scale=1.7, dtype=TYPES[to])
    assert Y.numel() * Y.element_size() >= HINT
    for part in parts(n, 5):
        assert torch.equal(Y[part], M.maxsim_embed(W, tokens[part], scale=1.7, dtype=TYPES[to]))
    R.check("Y", Y[-500:], T.embed(W, tokens[-500:], 1.7, TYPES[to]))


@pytest.mark.parametrize("dtype,to,n,vocab,d,accumulate", [("bf16", "f32", 40_000, 50_001, 1030, False), ("f32", "f32", 30_001, 40_003, 1201, False), ("f16", "f16", 300_000, 10_001, 512, True), ("bf16", "bf16", 8000, 100_003, 1284, True)])
def test_embed_backward(dtype, to, n, vocab, d, accumulate):
    print(dtype, to, n, vocab, d, accumulate, flush=True)
    dY, old = randn(n, d, seed=3, dtype=dtype), randn(vocab, d, seed=4, dtype=to)
    u = torch.rand(n, generator=gen(5), device=DEV)
    tokens = (u ** 4 * (vocab + 10)).long()  # (frequent ones, and some outside)
    out = old.clone()
    assert dY.numel() * dY.element_size() + out.numel() * out.element_size() >= HINT
    M.maxsim_embed_backward(dY, tokens, vocab, out=out, accumulate=accumulate, scale=0.5)
    torch.cuda.synchronize()
    R.check("dW", out, T.embed_backward(dY, tokens, vocab, 0.5, TYPES[to], old if accumulate else None))


# pieces of eight entries of 16 bits, four, two; of four and two of 32 bits; more than a wavefront's
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,d,rot", [("bf16", 128, 128), ("f16", 128, 96), ("f16", 80, 40), ("bf16", 84, 4), ("bf16", 84, 20), ("f32", 64, 64), ("f32", 84, 4)])
def test_norm_rope(dtype, d, rot, interleaved):
    print(dtype, d, rot, interleaved, flush=True)
    size, heads = TYPES[dtype].itemsize, 6
    n = HINT // (2 * heads * d * size) + 101
    X, dY, w = odd(n, heads, d, seed=6, dtype=dtype), odd(n, heads, d, seed=7, dtype=dtype), 1 + 0.1 * randn(2, d, seed=8)
    at = torch.randint(0, 5000, (n,), generator=gen(9), device=DEV, dtype=torch.int32)
    freqs = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float32) / rot)
    how = dict(q_heads=4, interleaved=interleaved, scale=1.1)
    Y = M.maxsim_norm_rope(X, freqs, w[0], w[1], positions=at, **how)
    dX, *dw = M.maxsim_norm_rope_backward(X, dY, freqs, w[0], w[1], positions=at, **how)
    total = [0.0, 0.0]
    for part in parts(n, 3):
        assert torch.equal(Y[part], M.maxsim_norm_rope(X[part], freqs, w[0], w[1], positions=at[part], **how))
        dx, *dws = M.maxsim_norm_rope_backward(X[part], dY[part], freqs, w[0], w[1], positions=at[part], **how)
        assert torch.equal(dX[part], dx)
        total = [a + b.double() for a, b in zip(total, dws)]
    R.check("Y", Y[-200:], T.norm_rope(X[-200:], freqs, w[0], w[1], 4, 1e-6, at[-200:], interleaved, 1.1))
    for part in (slice(0, 200), slice(n - 200, n)):
        R.check("dX", dX[part], T.norm_rope_backward(X[part], dY[part], freqs, w[0], w[1], 4, 1e-6, at[part], interleaved, 1.1)[0])
    # dw: sums of as many terms as there are rows, whose size is that of the terms: both ways within the bound of the definition's test, for all rows a part at a time
    for name, got, k in (("dq_weight", dw[0], 1), ("dk_weight", dw[1], 2)):
        value, terms = 0.0, 0.0
        for part in parts(n, 8):
            v, bound = T.norm_rope_backward(X[part], dY[part], freqs, w[0], w[1], 4, 1e-6, at[part], interleaved, 1.1)[k]
            value, terms = value + v, terms + bound * (n / (part.stop - part.start))  # (a bound has as many roundings as its rows, 64 more and the rotation's)
        R.check(name, got, (value, terms))
        R.check(name, total[k - 1], (value, terms))


# rows in a workgroup's registers, by its pieces, and rows read twice; parts of a call have enough rows for the same kernels
@pytest.mark.parametrize("dtype,n,b", [("bf16", 40_001, 4001), ("f16", 30_001, 6001), ("bf16", 14_001, 12_003), ("f32", 9001, 12_001), ("bf16", 3500, 50_001), ("f32", 2500, 30_005), ("bf16", 2500, 70_003), ("f32", 1500, 70_001)])
def test_distill(dtype, n, b):
    print(dtype, n, b, flush=True)
    k, size = 20, TYPES[dtype].itemsize
    scores, teacher = odd(n, b, seed=10, dtype=dtype), randn(n, k, seed=11)
    index = torch.randint(-1, b + 1, (n, k), generator=gen(12), device=DEV, dtype=torch.int32)
    up = torch.rand(n, generator=gen(13), device=DEV)
    assert n * b * size >= HINT
    loss, lse = M.maxsim_distill(scores, teacher, index, tau=0.7)
    back = M.maxsim_distill_backward(scores, teacher, lse, up, index, tau=0.7)
    g, loss2 = M.maxsim_distill_grad(scores, teacher, index, tau=0.7, weight=0.3)
    for part in parts(n, 1 + 2 * n * b * size // HINT):
        assert part.stop - part.start >= 256 and 2 * (part.stop - part.start) * b * size < HINT
        s, t, i = scores[part], teacher[part], index[part]
        a, c = M.maxsim_distill(s, t, i, tau=0.7)
        assert torch.equal(loss[part], a) and torch.equal(lse[part], c)
        assert torch.equal(back[part], M.maxsim_distill_backward(s, t, c, up[part], i, tau=0.7))
        a, c = M.maxsim_distill_grad(s, t, i, tau=0.7, weight=0.3)
        assert torch.equal(g[part], a) and torch.equal(loss2[part], c)
    for part in (slice(0, 30), slice(n - 30, n)):
        want = T.distill(scores[part], teacher[part], index[part], 0.7, up[part])
        R.check("loss", loss[part], want["loss"])
        R.check("g", back[part], want["g"])
