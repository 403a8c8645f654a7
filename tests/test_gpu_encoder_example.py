"""The example's training steps: attention, MaxSim, their gradients and the clipping work together, and the loss falls."""
import importlib.util
import os

import pytest
import torch

from paper_2605_29517_amd.rope import rope_frequencies

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_encoder", os.path.join(ROOT, "examples", "train_encoder.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_loss_falls(example):
    seen = example.train(24)
    first, last = (sum(loss for loss, _ in part) / 4 for part in (seen[:4], seen[-4:]))
    print("loss %.3f -> %.3f" % (first, last), flush=True)
    assert last < 0.8 * first
    assert all(norm > 0 for _, norm in seen)
    assert example.train(3) == example.train(3)  # the same bits again


def test_the_encoder_against_plain_operations(example):
    """Embeddings of the same texts, text by text in fp32. The rows differ by the roundings of 16-bit projections (2^-8 each, a handful of
    them on the way to a row of unit length)."""
    p = example.parameters(3)
    docs, offsets, _, _ = example.batch(5)
    freqs, _ = rope_frequencies(example.D, device="cuda")
    got = example.encode(p, docs, offsets, freqs).float()
    H, KV, d = example.HEADS, example.KV_HEADS, example.D
    for a, b in zip(offsets.tolist(), offsets.tolist()[1:]):
        x = p["tokens"][docs[a:b]].float()
        qkv = (x @ p["qkv"].t()).view(b - a, H + 2 * KV, d)
        angle = torch.arange(b - a, device="cuda").float()[:, None] * freqs
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        z = torch.complex(qkv[:, :H + KV, :d // 2].contiguous(), qkv[:, :H + KV, d // 2:].contiguous()) * turn
        qk = torch.cat((z.real, z.imag), -1)
        k, v = (t.repeat_interleave(H // KV, 1).transpose(0, 1) for t in (qk[:, H:], qkv[:, H + KV:]))
        w = torch.softmax(qk[:, :H].transpose(0, 1) @ k.transpose(1, 2).contiguous() / d ** 0.5, -1)
        x = x + (w @ v).transpose(0, 1).reshape(b - a, H * d) @ p["mix"].t()
        want = torch.nn.functional.normalize(x @ p["out"].t(), dim=-1)
        assert (got[a:b] - want).norm(dim=-1).max() < 8 * 2.0 ** -8
