"""Attention over packed sequences, its gradient and rotary positions from their definitions in 64 bits, with bounds on what 16-bit
operands may cost: shared by the tests of the kernels (tensors on the GPU) and of the formulas (on the CPU)."""
import math

import torch

# half a unit in the last place, relative; and half the distance of the smallest numbers
UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}


def allowed(lq, lk, causal, device):
    """Which keys a query sees, [lq, lk]."""
    i, j = torch.arange(lq, device=device)[:, None], torch.arange(lk, device=device)
    return j <= i + (lk - lq) if causal else torch.ones(lq, lk, dtype=torch.bool, device=device)


def pieces(q_off, k_off):
    q, k = q_off.tolist(), k_off.tolist()
    return zip(q, q[1:], k, k[1:])


def probabilities(q, k, mask, scale):
    """P and lse of one sequence and head; a row that sees nothing: zeros and -inf."""
    s = torch.where(mask, (q @ k.t()) * scale, -math.inf)
    top = s.amax(1, keepdim=True) if s.shape[1] else torch.full((s.shape[0], 1), -math.inf, dtype=s.dtype, device=s.device)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = torch.exp(s - top)
    total = e.sum(1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total), (top + torch.log(total))[:, 0]


def attention(Q, K, V, q_off, k_off, causal, scale, dO=None):
    """Results and, in step with each, a bound on the error of a computation with fp32 sums that rounds P, dS and its outputs to Q's type
    and takes delta from its own O: {"O": (value, bound), "lse": ..., "dQ", "dK", "dV"}."""
    u, tiny = UNIT[Q.dtype], TINY[Q.dtype]
    sums = 2e-6  # fp32 sums and exponentials: some 2^-24 each, of numbers that mostly do not agree in sign
    group = Q.shape[1] // K.shape[1]
    Q, K, V = Q.double(), K.double(), V.double()
    dO = None if dO is None else dO.double()
    zero = lambda t: (torch.zeros_like(t), torch.zeros_like(t))  # noqa: E731
    out = {"O": zero(Q), "lse": (torch.full(Q.shape[:2], -math.inf, dtype=torch.float64, device=Q.device), torch.zeros(Q.shape[:2], dtype=torch.float64, device=Q.device))}
    if dO is not None:
        out.update(dQ=zero(Q), dK=zero(K), dV=zero(V))
    for a, b, c, e in pieces(q_off, k_off):
        if a == b or c == e:
            continue
        mask = allowed(b - a, e - c, causal, Q.device)
        for h in range(Q.shape[1]):
            q, k, v = Q[a:b, h], K[c:e, h // group], V[c:e, h // group]
            p, lse = probabilities(q, k, mask, scale)
            o = p @ v
            # scores: an error of a few 2^-24 of the sum of |q k|, which P takes as a relative one
            ds_abs = (q.abs() @ k.abs().t()) * scale * 2.0 ** -22 + 2.0 ** -20
            p_err = p * (u + ds_abs) + tiny
            o_err = p_err @ v.abs() + sums * (p @ v.abs())
            out["O"][0][a:b, h], out["O"][1][a:b, h] = o, o_err + u * (o.abs() + o_err) + tiny
            out["lse"][0][a:b, h], out["lse"][1][a:b, h] = lse, (ds_abs * mask).amax(1) + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0)
            if dO is None:
                continue
            g = dO[a:b, h]
            dp = g @ v.t()
            delta = (g * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            delta_err = (g.abs() * out["O"][1][a:b, h]).sum(1, keepdim=True) + sums * (g * o).abs().sum(1, keepdim=True)
            dp_err = sums * (g.abs() @ v.abs().t())
            p32 = p * ds_abs
            ds_err = ds.abs() * u + tiny + (p * (delta_err + dp_err) + p32 * (dp - delta).abs()) * (1 + u)
            for name, value, err in (("dQ", ds @ k * scale, (ds_err + sums * ds.abs()) @ k.abs() * scale),
                                     ("dK", ds.t() @ q * scale, (ds_err + sums * ds.abs()).t() @ q.abs() * scale),
                                     ("dV", p.t() @ g, (p_err + sums * p).t() @ g.abs())):
                at = (slice(a, b), h) if name == "dQ" else (slice(c, e), h // group)
                out[name][0][at] += value
                out[name][1][at] += err
    for name in ("dQ", "dK", "dV"):
        if name in out:
            value, err = out[name]
            err += u * (value.abs() + err) + tiny
    return out


def check(name, got, want):
    """got within the bound of want = (value, bound), infinities alike."""
    value, bound = want
    got = got.double()
    finite = torch.isfinite(value)
    assert torch.equal(got[~finite], value[~finite]), "%s: infinities differ" % name
    off = (got[finite] - value[finite]).abs()
    assert torch.isfinite(got[finite]).all(), "%s: not finite" % name
    over = off > bound[finite]
    assert not over.any(), "%s: %d of %d beyond the bound, the worst %.3g times" % (name, int(over.sum()), over.numel(), float((off / bound[finite].clamp_min(1e-300)).max()))


def rope(X, freqs, at, interleaved, inverse, scale):
    """Rotary positions by complex products in 64 bits."""
    rot = 2 * freqs.shape[0]
    angle = at.double()[:, None] * freqs.double()
    turn = torch.polar(torch.full_like(angle, scale), -angle if inverse else angle)[:, None]
    out = X.double().clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(out[..., first].contiguous(), out[..., second].contiguous()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def offsets(lengths, device):
    off = torch.zeros(len(lengths) + 1, dtype=torch.int64)
    off[1:] = torch.cumsum(torch.tensor(lengths, dtype=torch.int64), 0)
    return off.to(torch.int32).to(device)
