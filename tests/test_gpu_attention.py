"""maxsim_attention and maxsim_attention_backward against their definitions in 64 bits, element by element within bounds that follow
from the roundings they make (attention_reference.py)."""
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
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def inputs(q_lens, k_lens, hq, hkv, d, dtype, seed=0, by=2.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    make = lambda t, h, x=1.0: (torch.randn(t, h, d, generator=g, device=DEV) * x).to(TYPES[dtype])  # noqa: E731
    tq, tk = sum(q_lens), sum(k_lens)
    return make(tq, hq, by), make(tk, hkv), make(tk, hkv), make(tq, hq), R.offsets(q_lens, DEV), R.offsets(k_lens, DEV)


def run(Q, K, V, dO, qo, ko, causal, scale=None):
    O, lse = M.maxsim_attention(Q, K, V, qo, ko, causal=causal, scale=scale)
    dQ, dK, dV = M.maxsim_attention_backward(Q, K, V, O, lse, dO, qo, ko, causal=causal, scale=scale)
    torch.cuda.synchronize()
    return {"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV}


def compare(case, Q, K, V, dO, qo, ko, causal, scale=None):
    print(case, flush=True)
    got = run(Q, K, V, dO, qo, ko, causal, scale)
    want = R.attention(Q, K, V, qo, ko, causal, Q.shape[2] ** -0.5 if scale is None else scale, dO)
    for name in want:
        R.check(name, got[name], want[name])
    return got


LENGTHS = {
    "one token": ([1], [1]),
    "tile edges": ([31, 32, 33, 63, 64, 65, 127, 128, 129], None),
    "odd and empty": ([0, 5, 0, 0, 300, 1, 77, 0], None),
    "one long": ([1000], None),
    "single tokens": ([1, 1, 1, 1, 1], [1, 63, 700, 0, 64]),
    "appended": ([3, 40, 130, 7], [50, 333, 130, 1000]),
    "more queries than keys": ([10, 200, 65, 4], [3, 70, 0, 5]),  # causal: rows that see nothing
    "many short": ([7, 2, 11, 1] * 40, None),
}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 4, 2, 128), ("f16", 3, 3, 64)])
def test_lengths(lengths, dtype, hq, hkv, d, causal):
    q, k = LENGTHS[lengths]
    compare((lengths, dtype, hq, hkv, d, causal), *inputs(q, q if k is None else k, hq, hkv, d, dtype), causal)


@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 48, 56, 72, 80, 88, 96, 104, 112, 120, 128, 136, 160, 200, 248, 256])
def test_widths(d):
    compare(d, *inputs([70, 9, 130], [70, 200, 131], 2, 1, d, "bf16" if d % 16 else "f16"), True)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (6, 2), (5, 5), (71, 1), (20, 4)])
def test_heads(hq, hkv):
    compare((hq, hkv), *inputs([40, 1, 150], [40, 90, 150], hq, hkv, 64, "bf16"), True)


@pytest.mark.parametrize("b,lq,lk,hq,hkv,d", [(1, 1, 20011, 4, 1, 128), (3, 1, 5000, 8, 2, 64), (2, 30, 4097, 2, 2, 96), (1, 2, 700, 1, 1, 32), (2, 1, 3001, 8, 1, 256)])
def test_few_queries_many_keys(b, lq, lk, hq, hkv, d):
    """Where the keys are taken in pieces."""
    for causal in (True, False):
        compare((b, lq, lk, causal), *inputs([lq] * b, [lk - 17 * i for i in range(b)], hq, hkv, d, "bf16"), causal)


@pytest.mark.parametrize("q,k,hq,hkv,d,dtype", [
    ([1, 1, 1, 2, 1], [24000, 1, 0, 700, 333], 32, 8, 128, "bf16"),
    ([1] * 5, [8000, 8001, 8191, 33, 8500], 8, 8, 96, "f16"),
    ([2, 3, 1], [20000, 13001, 64], 12, 12, 64, "f16"),
    ([1], [50000], 16, 16, 32, "bf16"),
    ([1, 0, 1], [6000, 9000, 29000], 16, 8, 72, "bf16"),
    ([4, 1], [12000, 700], 16, 8, 256, "f16"),
    ([1, 1], [65537, 131000], 32, 1, 128, "f16"),
    ([30], [24500], 8, 8, 128, "bf16"),
])
def test_few_queries_large_caches(q, k, hq, hkv, d, dtype):
    """From 100 MB of keys and values on they stream past the caches, to a wavefront of its own for every second tile."""
    assert sum(k) * hkv * d * 4 >= 1e8 and sum(q) * (hq // hkv) <= 32 * len(q)
    Q, K, V, _, qo, ko = inputs(q, k, hq, hkv, d, dtype)
    for causal in (True, False):
        print(q, k, hq, hkv, d, dtype, causal, flush=True)
        O, lse = M.maxsim_attention(Q, K, V, qo, ko, causal=causal)
        torch.cuda.synchronize()
        want = R.attention(Q, K, V, qo, ko, causal, d ** -0.5)
        R.check("O", O, want["O"])
        R.check("lse", lse, want["lse"])


@pytest.mark.parametrize("lens,hq,hkv,d", [([1000], 8, 1, 128), ([700, 33], 6, 2, 80), ([2000], 1, 1, 64), ([129, 0, 1500], 16, 1, 32), ([700, 5], 8, 1, 256)])
def test_few_key_heads(lens, hq, hkv, d):
    """Where the queries of a key tile are taken in pieces for dK and dV."""
    for causal in (True, False):
        compare((lens, hq, hkv, d, causal), *inputs(lens, lens, hq, hkv, d, "bf16"), causal)
    compare("other queries", *inputs([3 * n for n in lens], lens, hq, hkv, d, "f16"), True)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,d,dtype", [(40, 64, "bf16"), (128, 64, "f16"), (200, 128, "bf16"), (700, 64, "bf16"), (1500, 128, "f16")])
def test_errors_in_the_norm(n, d, dtype, causal):
    """Where every result is rounded once and one operand of its sum once (P for O and dV, dS for dK and dQ), both by u at random, the error is
    sqrt(2) of what the rounding of the results alone makes; half as much again of that second rounding is left for delta: 1.5."""
    Q, K, V, dO, qo, ko = inputs([n] * (1 + 300 // n), [n] * (1 + 300 // n), 8, 2, d, dtype)
    got = run(Q, K, V, dO, qo, ko, causal)
    want = R.attention(Q, K, V, qo, ko, causal, d ** -0.5, dO)
    for name in ("O", "dQ", "dK", "dV"):
        value = want[name][0]
        alone = (value.to(Q.dtype).double() - value).norm()
        off = (got[name].double() - value).norm()
        print(n, d, dtype, causal, name, "%.3f" % float(off / alone), flush=True)
        assert off <= 1.5 * alone, name


def test_small_gradients():
    """fp16 gradients of 10^-3: P and dS leave the range of normal numbers, which the bounds count."""
    Q, K, V, dO, qo, ko = inputs([300, 20], [300, 20], 4, 2, 64, "f16")
    compare("small", Q, K, V, dO * 2.0 ** -10, qo, ko, True)


def test_scale_and_sharp_rows():
    """Another scale, and scores of some hundreds: rows that look at one token."""
    compare("scale", *inputs([100, 50], [100, 50], 2, 2, 64, "f16"), True, scale=0.3)
    compare("sharp", *inputs([200], [200], 2, 2, 64, "bf16", by=60.0), False)


def test_views():
    """Slices of one projection [tokens, (hq + 2 hkv) d], heads before tokens, outputs into a slice."""
    hq, hkv, d, lens = 4, 2, 64, [90, 33, 200]
    Q, K, V, dO, qo, ko = inputs(lens, lens, hq, hkv, d, "bf16")
    want = run(Q, K, V, dO, qo, ko, True)
    fused = torch.cat((Q, K, V), 1)
    q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    t = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    grads = torch.full_like(fused, float("nan"))
    room = torch.full((sum(lens), 2 * hq, d), float("nan"), device=DEV, dtype=Q.dtype)
    for a, b, c, g in ((q, k, v, dO), (t(Q), t(K), t(V), t(dO)), (q, t(K), v, t(dO))):
        O, lse = M.maxsim_attention(a, b, c, qo, ko, out=room[:, 1:hq + 1])
        dQ, dK, dV = M.maxsim_attention_backward(a, b, c, O, lse, g, qo, ko, dQ=grads[:, :hq], dK=grads[:, hq:hq + hkv], dV=grads[:, hq + hkv:])
        torch.cuda.synchronize()
        for name, x in (("O", O), ("lse", lse), ("dQ", dQ), ("dK", dK), ("dV", dV)):
            assert torch.equal(x, want[name]), name
        assert torch.isnan(room[:, 0]).all() and torch.isnan(room[:, hq + 1:]).all()


def test_one_head_for_all_is_a_broadcast_view():
    """K and V of one head, expanded to as many as Q has: the same results as shared heads, and no gradient may go into such a view."""
    Q, K, V, dO, qo, ko = inputs([100, 20], [100, 20], 4, 1, 64, "f16")
    O, lse = M.maxsim_attention(Q, K, V, qo, ko)
    O2, lse2 = M.maxsim_attention(Q, K.expand(-1, 4, -1), V.expand(-1, 4, -1), qo, ko)
    torch.cuda.synchronize()
    R.check("O", O2, (O.double(), 2 * R.UNIT[Q.dtype] * (O.double().abs() + 1)))
    assert torch.allclose(lse, lse2, rtol=1e-5, atol=1e-5)
    with pytest.raises(M.MaxSimError, match="invalid"):
        M.maxsim_attention_backward(Q, K.expand(-1, 4, -1), V.expand(-1, 4, -1), O, lse, dO, qo, ko, dK=torch.empty_like(K).expand(-1, 4, -1))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_sequence_does_not_reach_another(bad):
    """Rows of one sequence that are not finite leave the others' results as they are, bit by bit."""
    lens = [50, 13, 90, 64]
    Q, K, V, dO, qo, ko = inputs(lens, lens, 2, 1, 64, "bf16")
    want = run(Q, K, V, dO, qo, ko, True)
    rows = slice(50, 63)
    for t in (Q, K, V, dO):
        t[rows] = bad
    got = run(Q, K, V, dO, qo, ko, True)
    keep = torch.ones(sum(lens), dtype=torch.bool, device=DEV)
    keep[rows] = False
    for name in want:
        assert torch.equal(got[name][keep], want[name][keep]), name


def test_the_same_bits_again():
    args = inputs([700, 30, 900], [700, 30, 900], 8, 2, 128, "bf16")
    a, b = run(*args, True), run(*args, True)
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_outputs_are_fully_written():
    """Memory that held NaNs before: sequences without keys or without queries too."""
    Q, K, V, dO, qo, ko = inputs([5, 0, 40, 3], [0, 70, 40, 200], 2, 2, 64, "f16")
    nan = lambda t: torch.full_like(t, float("nan"))  # noqa: E731
    O, lse = M.maxsim_attention(Q, K, V, qo, ko, out=nan(Q), lse=torch.full(Q.shape[:2], float("nan"), device=DEV))
    grads = M.maxsim_attention_backward(Q, K, V, O, lse, dO, qo, ko, dQ=nan(Q), dK=nan(K), dV=nan(V))
    torch.cuda.synchronize()
    assert not O.isnan().any() and not lse.isnan().any() and not any(g.isnan().any() for g in grads)
    assert (O[:5] == 0).all() and (lse[:5] == -math.inf).all() and (grads[0][:5] == 0).all() and (grads[1][:70] == 0).all()


def test_rows_far_apart():
    """A sequence whose rows span more than 4 GiB: 300 rows, 2^24 - 8 entries from one to the next."""
    lens, stride, d = [300], (1 << 24) - 8, 64
    Q, K, V, dO, qo, ko = inputs(lens, lens, 1, 1, d, "bf16")
    far = torch.empty(300 * stride, dtype=Q.dtype, device=DEV).as_strided((300, 3, d), (stride, 4096, 1))
    far[:, 0:1], far[:, 1:2], far[:, 2:3] = Q, K, V
    want = run(Q, K, V, dO, qo, ko, True)
    got = run(far[:, 0:1], far[:, 1:2], far[:, 2:3], dO, qo, ko, True)
    for name in want:
        assert torch.equal(got[name], want[name]), name


def test_on_another_stream():
    Q, K, V, dO, qo, ko = inputs([600, 100], [600, 100], 4, 2, 64, "bf16")
    want = run(Q, K, V, dO, qo, ko, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        q = Q * 1
        O, lse = M.maxsim_attention(q, K, V, qo, ko)
        dQ, dK, dV = M.maxsim_attention_backward(q, K, V, O, lse, dO, qo, ko)
    side.synchronize()
    for name, x in (("O", O), ("lse", lse), ("dQ", dQ), ("dK", dK), ("dV", dV)):
        assert torch.equal(x, want[name]), name


def test_autograd():
    """The differentiable form, with a loss whose gradient comes as an expanded view, and against differences of the loss."""
    lens = [40, 25]
    Q, K, V, _, qo, _ = inputs(lens, lens, 4, 2, 64, "f16", by=0.5)
    leaf = [t.clone().requires_grad_() for t in (Q, K, V)]
    A.attention(*leaf, qo).sum().backward()
    want = R.attention(Q, K, V, qo, qo, True, 64 ** -0.5, torch.ones_like(Q))
    for name, t in zip(("dQ", "dK", "dV"), leaf):
        R.check(name, t.grad, want[name])
    # differences along one direction: steps of 2^-5 are exact in the inputs up to rounding of their last bits, which the direction is read from
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    G = torch.randn(Q.shape, generator=g, device=DEV)
    leaf = [t.clone().requires_grad_() for t in (Q, K, V)]
    (A.attention(*leaf, qo).float() * G).sum().backward()
    for n, t in enumerate((Q, K, V)):
        step = torch.randn(t.shape, generator=g, device=DEV) * 2.0 ** -5
        up, down = (t + step).half(), (t - step).half()
        value = [(A.attention(*[x if m == n else y for m, y in enumerate((Q, K, V))], qo).double() * G).sum().item() for x in (up, down)]
        along = (leaf[n].grad.double() * (up.double() - down.double())).sum().item()
        # what roundings of O (2^-11 each, some 10^4 of them, without agreement) and the third derivative make of it
        size = (leaf[n].grad.double() * (up.double() - down.double())).norm().item()
        assert abs(value[0] - value[1] - along) < 0.05 * abs(along) + 0.05 * size + 0.1, (n, value[0] - value[1], along)


def test_graph():
    """Captured, and replayed on other inputs with the program's own work in between."""
    M.maxsim_init()
    lens = [100, 1, 260]
    args = inputs(lens, lens, 4, 2, 64, "bf16")
    Q, K, V, dO, qo, ko = args
    ws = torch.empty(M.load().maxsim_attention_backward_workspace(3, 361, 361, 4, 2, 64), dtype=torch.uint8, device=DEV)
    run(*args, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        O, lse = M.maxsim_attention(Q, K, V, qo, ko)
        grads = M.maxsim_attention_backward(Q, K, V, O, lse, dO, qo, ko, workspace=ws)
    for seed in range(3):
        fresh = inputs(lens, lens, 4, 2, 64, "bf16", seed=seed + 50)
        for t, f in zip((Q, K, V, dO), fresh):
            t.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (O, lse, *grads)]
        want = run(*args, True)
        for x, name in zip(got, ("O", "lse", "dQ", "dK", "dV")):
            assert torch.equal(x, want[name]), (seed, name)


def test_refusals():
    Q, K, V, dO, qo, ko = inputs([10], [10], 4, 2, 64, "f16")
    with pytest.raises(M.MaxSimError, match="dtype"):
        M.maxsim_attention(Q.float(), K.float(), V.float(), qo)
    with pytest.raises(M.MaxSimError, match="dtype"):
        M.maxsim_attention(Q, K.bfloat16(), V, qo)
    with pytest.raises(M.MaxSimError, match="divides"):
        M.maxsim_attention(Q[:, :3].contiguous(), K, V, qo)
    with pytest.raises(M.MaxSimError, match="offsets"):
        M.maxsim_attention(Q, K, V, qo, torch.zeros(3, dtype=torch.int32, device=DEV))
    with pytest.raises(M.MaxSimError, match="same rows"):
        M.maxsim_attention(Q, K[:5], V[:5], qo)
    with pytest.raises(M.MaxSimError, match="dtype"):
        M.maxsim_attention(Q, K, V, qo.long())
    with pytest.raises(M.MaxSimError, match="must be on"):
        M.maxsim_attention(Q, K, V, qo.cpu())
    with pytest.raises(M.MaxSimError, match="unsupported|built"):
        M.maxsim_attention(*inputs([4], [4], 1, 1, 264, "f16")[:3], R.offsets([4], DEV))
    with pytest.raises(M.MaxSimError, match="invalid"):
        M.maxsim_attention(Q, K, V, qo, scale=0.0)
    with pytest.raises(M.MaxSimError, match="rows of stride 1"):
        M.maxsim_attention(Q.transpose(1, 2).contiguous().transpose(1, 2), K, V, qo)
    odd = torch.empty(10 * 4 * 64 + 1, dtype=Q.dtype, device=DEV)[1:].view(10, 4, 64)
    with pytest.raises(M.MaxSimError, match="invalid"):
        M.maxsim_attention(odd, K, V, qo)
    O, lse = M.maxsim_attention(Q, K, V, qo)
    with pytest.raises(M.MaxSimError, match="scratch|workspace"):
        M.maxsim_attention_backward(Q, K, V, O, lse, dO, qo, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(M.MaxSimError, match="lse"):
        M.maxsim_attention_backward(Q, K, V, O, lse[:, :2], dO, qo)
