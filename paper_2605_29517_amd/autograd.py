"""torch.autograd glue over the C ABI (marshalling only): the forward keeps the int32 argmax the kernels
emit (Sec. "Closed-Form Gradients"), the backward hands it with the upstream gradient to maxsim_backward.
Nothing is computed here; every step runs in the HIP kernels, and there is no CPU fallback.

Scores and attention can be differentiated once: to go on through a gradient that was made with create_graph=True raises an error (the
kernels leave no graph of it). Rotary positions are linear and can be differentiated any number of times."""
import torch
from torch.autograd.function import once_differentiable

from . import binding as M


def _once(backward):
    """once_differentiable where a graph of the gradient is asked for; elsewhere backward as it is (a microsecond of a small step)."""
    guarded = once_differentiable(backward)
    return lambda ctx, g: guarded(ctx, g) if torch.is_grad_enabled() else backward(ctx, g)


class _MaxSim(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, D):
        scores, argmax = M.maxsim_forward(Q, D, want_argmax=True)
        ctx.save_for_backward(Q, D, argmax)
        return scores

    @staticmethod
    @_once
    def backward(ctx, dscore):
        Q, D, argmax = ctx.saved_tensors
        dQ, dD = M.maxsim_backward(Q, D, argmax, dscore.contiguous().float())
        return dQ.to(Q.dtype), dD.to(D.dtype)


class _MaxSimRagged(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, D_packed, doc_offsets):
        scores, argmax = M.maxsim_forward_ragged(Q, D_packed, doc_offsets, want_argmax=True)
        ctx.save_for_backward(Q, D_packed, doc_offsets, argmax)
        return scores

    @staticmethod
    @_once
    def backward(ctx, dscore):
        Q, D_packed, doc_offsets, argmax = ctx.saved_tensors
        dQ, dD = M.maxsim_backward_ragged(Q, D_packed, doc_offsets, argmax, dscore.contiguous().float())
        return dQ.to(Q.dtype), dD.to(D_packed.dtype), None


def maxsim(Q, D, doc_offsets=None):
    """Differentiable scores [n_q, b] of Q [n_q,l_q,d] against D [b,l_d,d], or against a packed corpus
    D [T,d] with int32 doc_offsets [b+1] (all on the GPU; d as the forward and backward entry points take it).  An empty ragged document scores -inf and receives no gradient."""
    if doc_offsets is None:
        return _MaxSim.apply(Q, D)
    return _MaxSimRagged.apply(Q, D, doc_offsets)


def _rows(t):
    """t as the rotary entry point takes it fastest: rows of stride 1 in pieces of 16 bytes (a view if it is one of those)."""
    size = t.element_size()
    fine = t.dim() == 3 and t.stride(2) == 1 and (t.data_ptr() | t.stride(0) * size | t.stride(1) * size) % 16 == 0
    return t if fine else t.contiguous()


def _pieces(t):
    """t as the attention entry points take it: rows of stride 1 in pieces of 16 bytes, less than 2^24 entries apart (a view if it is one of
    those, otherwise a copy, also where t is contiguous but at an odd address)."""
    t = _rows(t)
    return t if t.data_ptr() % 16 == 0 and t.stride(0) < 1 << 24 else t.clone(memory_format=torch.contiguous_format)


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, freqs, positions, offsets, interleaved, scale, inverse):
        ctx.save_for_backward(freqs, positions, offsets)
        ctx.how = interleaved, scale, inverse
        return M.maxsim_rope(_rows(X), freqs, positions, offsets, interleaved=interleaved, scale=scale, inverse=inverse)

    @staticmethod
    def backward(ctx, dY):
        freqs, positions, offsets = ctx.saved_tensors
        interleaved, scale, inverse = ctx.how
        return (_Rope.apply(dY, freqs, positions, offsets, interleaved, scale, not inverse),) + (None,) * 6


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, q_offsets, k_offsets, causal, scale):
        Q, K, V = _pieces(Q), _pieces(K), _pieces(V)
        out, lse = M.maxsim_attention(Q, K, V, q_offsets, k_offsets, causal=causal, scale=scale)
        ctx.save_for_backward(Q, K, V, out, lse, q_offsets, k_offsets)
        ctx.how = causal, scale
        return out

    @staticmethod
    @_once
    def backward(ctx, dout):
        Q, K, V, out, lse, q_offsets, k_offsets = ctx.saved_tensors
        causal, scale = ctx.how
        return M.maxsim_attention_backward(Q, K, V, out, lse, _pieces(dout), q_offsets, k_offsets, causal=causal, scale=scale) + (None,) * 4


def rope(X, freqs, positions=None, offsets=None, interleaved=False, scale=1.0):
    """Differentiable rotary positions of X [tokens, heads, d] (binding.maxsim_rope; no gradient for freqs)."""
    return _Rope.apply(X, freqs, positions, offsets, interleaved, scale, False)


def attention(Q, K, V, q_offsets, k_offsets=None, causal=True, scale=None):
    """Differentiable attention over packed sequences (binding.maxsim_attention)."""
    return _Attention.apply(Q, K, V, q_offsets, k_offsets, causal, scale)
