"""The differentiable forms without a GPU: the entry points are replaced by plain operations, so that what is tested is the glue alone."""
import os
import sys

import pytest
import torch

from paper_2605_29517_amd import autograd as A

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import attention_reference as R  # noqa: E402

R.UNIT.setdefault(torch.float64, 2.0 ** -53)
R.TINY.setdefault(torch.float64, 0.0)


class Plain:
    """The entry points that the differentiable forms call, in 64 bits on the CPU."""

    @staticmethod
    def maxsim_rope(X, freqs, positions=None, offsets=None, interleaved=False, inverse=False, scale=1.0):
        at = positions if positions is not None else torch.arange(X.shape[0])
        return R.rope(X.detach(), freqs, at, interleaved, inverse, scale)

    @staticmethod
    def maxsim_attention(Q, K, V, q_offsets, k_offsets=None, causal=True, scale=None):
        out = R.attention(Q.detach(), K.detach(), V.detach(), q_offsets, q_offsets if k_offsets is None else k_offsets, causal, Q.shape[2] ** -0.5 if scale is None else scale)
        return out["O"][0], out["lse"][0]

    @staticmethod
    def maxsim_attention_backward(Q, K, V, out, lse, dout, q_offsets, k_offsets=None, causal=True, scale=None):
        got = R.attention(Q.detach(), K.detach(), V.detach(), q_offsets, q_offsets if k_offsets is None else k_offsets, causal, Q.shape[2] ** -0.5 if scale is None else scale, dout.detach())
        return got["dQ"][0], got["dK"][0], got["dV"][0]

    @staticmethod
    def maxsim_forward(Q, D, want_argmax=True):
        s = torch.einsum("qid,bjd->qbij", Q.detach(), D.detach())
        return s.amax(-1).sum(-1), s.argmax(-1).int()

    @staticmethod
    def maxsim_backward(Q, D, argmax, dscore):
        dQ, dD = torch.zeros_like(Q), torch.zeros_like(D)
        for q in range(Q.shape[0]):
            for b in range(D.shape[0]):
                for i in range(Q.shape[1]):
                    j = int(argmax[q, b, i])
                    dQ[q, i] += dscore[q, b].detach() * D[b, j].detach()
                    dD[b, j] += dscore[q, b].detach() * Q[q, i].detach()
        return dQ, dD


@pytest.fixture
def plain(monkeypatch):
    monkeypatch.setattr(A, "M", Plain)


def randn(*shape, seed=1):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_twice_differentiable(plain, interleaved):
    """Against differences, once and twice; a gradient penalty reaches its inputs."""
    freqs, at = torch.tensor([0.5, 0.1], dtype=torch.float64), torch.tensor([0, 3, 7, 2, 9], dtype=torch.int32)
    f = lambda x: A.rope(x, freqs, positions=at, interleaved=interleaved, scale=1.3)  # noqa: E731
    X = randn(5, 2, 6).requires_grad_()
    assert torch.autograd.gradcheck(f, (X,))
    assert torch.autograd.gradgradcheck(f, (X,))
    g, = torch.autograd.grad((f(X) ** 3).sum(), X, create_graph=True)
    assert g.grad_fn is not None and torch.autograd.grad(g.square().sum(), X)[0].abs().max() > 0


def test_attention_and_maxsim_refuse_second_derivatives(plain):
    """The first derivative is there with create_graph too; to go on through it is an error and not a gradient that is silently missing."""
    off = torch.tensor([0, 3, 7], dtype=torch.int32)
    Q, K, V = (randn(7, 2, 4, seed=s).requires_grad_() for s in (1, 2, 3))
    assert torch.autograd.gradcheck(lambda *x: A.attention(*x, off), (Q, K, V))
    grads = torch.autograd.grad(A.attention(Q, K, V, off).square().sum(), (Q, K, V), create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (Q.sum() + grads[0].square().sum()).backward()
    Q, D = randn(2, 3, 4).float().requires_grad_(), randn(3, 5, 4, seed=2).float().requires_grad_()
    grads = torch.autograd.grad(A.maxsim(Q, D).square().sum(), (Q, D), create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (Q.sum() + grads[1].square().sum()).backward()


def acceptable(t):
    """What the C side asks of a tensor's address and strides (in elements of 16 bits)."""
    token, head = t.stride(0) if t.shape[0] > 1 else t.shape[2], t.stride(1) if t.shape[1] > 1 else t.shape[2]
    return t.stride(2) == 1 and t.data_ptr() % 16 == 0 and token % 8 == 0 and head % 8 == 0 and token < 1 << 24


def odd(shape, by):
    """A contiguous view at an address that is no multiple of 16 bytes."""
    flat = torch.randn(torch.Size(shape).numel() + by, generator=torch.Generator().manual_seed(5)).half()
    return flat[by:].view(shape)


LAYOUTS = {
    "odd address": lambda: odd((6, 2, 8), 1),
    "slice of odd rows": lambda: odd((6, 2, 12), 0)[:, :, :8],
    "innermost not 1": lambda: odd((6, 8, 2), 0).transpose(1, 2),
    "expanded": lambda: odd((1, 1, 1), 0).expand(6, 2, 8),
    "rows too far apart": lambda: torch.zeros(5 * (1 << 24) + 16, dtype=torch.float16).as_strided((6, 2, 8), (1 << 24, 8, 1)),
    "fitting view": lambda: odd((6, 4, 8), 0)[:, 1:3],
}


@pytest.mark.parametrize("layout", LAYOUTS)
def test_attention_of_any_layout(monkeypatch, layout):
    """Inputs and upstream gradients that the kernels do not take as they lie are copied; what they do take is not."""
    seen = []

    class Entry(Plain):
        @staticmethod
        def maxsim_attention(Q, K, V, *a, **k):
            seen.extend((Q, K, V))
            return torch.zeros(Q.shape, dtype=Q.dtype), torch.zeros(Q.shape[:2])

        @staticmethod
        def maxsim_attention_backward(Q, K, V, out, lse, dout, *a, **k):
            seen.append(dout)
            return torch.zeros(Q.shape).half(), torch.zeros(K.shape).half(), torch.zeros(V.shape).half()

    monkeypatch.setattr(A, "M", Entry)
    t = LAYOUTS[layout]()
    leaf = t.detach().clone().requires_grad_()
    out = A.attention(t, t, leaf, torch.tensor([0, 6], dtype=torch.int32))
    out.backward(LAYOUTS[layout]())
    assert len(seen) == 4
    for x in seen:
        assert acceptable(x) and torch.equal(x, t), (layout, x.stride(), x.data_ptr() % 16)
    if layout == "fitting view":
        assert seen[0] is t or seen[0].data_ptr() == t.data_ptr()
