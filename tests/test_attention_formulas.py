"""The 64-bit definitions that the GPU tests of attention and rotary positions compare with: against brute force and differences, and the
frequencies of long contexts (no GPU needed)."""
import math
import os
import sys

import pytest
import torch

from paper_2605_29517_amd.rope import rope_frequencies

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import attention_reference as R  # noqa: E402


def inputs(q_lens, k_lens, hq=4, hkv=2, d=6):
    g = torch.Generator().manual_seed(1)
    make = lambda t, h: torch.randn(t, h, d, generator=g, dtype=torch.float64)  # noqa: E731
    return make(sum(q_lens), hq), make(sum(k_lens), hkv), make(sum(k_lens), hkv), make(sum(q_lens), hq), R.offsets(q_lens, "cpu"), R.offsets(k_lens, "cpu")


R.UNIT[torch.float64], R.TINY[torch.float64] = 2.0 ** -53, 0.0


@pytest.mark.parametrize("causal", [False, True])
def test_forward_by_loops(causal):
    q_lens, k_lens = [3, 0, 5, 4], [3, 4, 2, 0]
    Q, K, V, _, qo, ko = inputs(q_lens, k_lens)
    out = R.attention(Q, K, V, qo, ko, causal, 0.4)
    for s, (lq, lk) in enumerate(zip(q_lens, k_lens)):
        for i in range(lq):
            for h in range(4):
                row, kv = int(qo[s]) + i, h // 2
                keys = [j for j in range(lk) if not causal or j <= i + lk - lq]
                score = [0.4 * float(Q[row, h] @ K[int(ko[s]) + j, kv]) for j in keys]
                total = sum(math.exp(x) for x in score)
                lse = math.log(total) if keys else -math.inf
                want = sum((math.exp(x) / total * V[int(ko[s]) + j, kv] for x, j in zip(score, keys)), torch.zeros(6, dtype=torch.float64))
                assert torch.allclose(out["O"][0][row, h], want, atol=1e-12)
                assert float(out["lse"][0][row, h]) == pytest.approx(lse, abs=1e-12)


@pytest.mark.parametrize("causal", [False, True])
def test_gradients_by_differences(causal):
    q_lens, k_lens = [4, 6], [7, 3]
    Q, K, V, G, qo, ko = inputs(q_lens, k_lens)

    def loss(*qkv):
        return float((R.attention(*qkv, qo, ko, causal, 0.4)["O"][0] * G).sum())

    out = R.attention(Q, K, V, qo, ko, causal, 0.4, G)
    g = torch.Generator().manual_seed(2)
    for n, name in enumerate(("dQ", "dK", "dV")):
        args = [Q, K, V]
        step = 1e-5 * torch.randn(args[n].shape, generator=g, dtype=torch.float64)
        up, down = (loss(*[x + s * step if m == n else x for m, x in enumerate(args)]) for s in (1, -1))
        assert (up - down) / 2 == pytest.approx(float((out[name][0] * step).sum()), rel=1e-6, abs=1e-11)


def test_rope_is_a_rotation_and_its_inverse():
    g = torch.Generator().manual_seed(3)
    X = torch.randn(9, 2, 12, generator=g, dtype=torch.float64)
    freqs, at = rope_frequencies(8)[0], torch.arange(9) * 1000
    for interleaved in (False, True):
        Y = R.rope(X, freqs, at, interleaved, False, 1.0)
        assert torch.allclose(Y.norm(dim=-1), X.norm(dim=-1)) and torch.equal(Y[..., 8:], X[..., 8:]) and torch.equal(Y[0], X[0])
        assert torch.allclose(R.rope(Y, freqs, at, interleaved, True, 1.0), X)
        # products of turned rows depend on the distance alone
        Z = R.rope(X[:1].expand(9, -1, -1), freqs, at + 17, interleaved, False, 1.0)
        W = R.rope(X[:1].expand(9, -1, -1), freqs, at + 5, interleaved, False, 1.0)
        dots = (Z * W).sum(-1)
        assert torch.allclose(dots, dots[:1].expand(9, -1))


def test_frequencies():
    plain, one = rope_frequencies(64)
    assert one == 1.0 and plain.dtype == torch.float32 and plain.shape == (32,) and float(plain[0]) == 1.0
    assert float(plain[-1]) == pytest.approx(10000.0 ** (-62 / 64))
    assert torch.allclose(rope_frequencies(64, factor=4.0, scaling="linear")[0], plain / 4)
    grown = rope_frequencies(64, factor=4.0, scaling="base")[0]
    assert float(grown[0]) == 1.0 and float(grown[-1]) == pytest.approx(float(plain[-1]) / 4, rel=1e-6)
    parts, scale = rope_frequencies(64, factor=8.0, scaling="parts", original=2048)
    turns = 2048 * plain.double() / (2 * math.pi)
    assert scale == pytest.approx(0.1 * math.log(8.0) + 1.0)
    assert torch.equal(parts[turns >= 40], plain[turns >= 40])
    assert torch.allclose(parts[turns <= 0.9], plain[turns <= 0.9] / 8)
    assert (parts <= plain).all() and (parts >= plain / 8 * (1 - 1e-6)).all()
    assert torch.equal(rope_frequencies(64, factor=1.0, scaling="parts")[0], plain)
    for bad in (dict(rot=3), dict(rot=64, factor=0.5), dict(rot=64, factor=2.0, scaling="other"), dict(rot=2, factor=2.0, scaling="base")):
        with pytest.raises(ValueError):
            rope_frequencies(**bad)
