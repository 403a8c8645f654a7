#!/usr/bin/env python3
"""Training steps of a small late-interaction encoder whose hot operators are all the library's: rotary positions and attention over
packed texts, MaxSim between every query and every document, the cross-entropy over in-batch negatives, the gradients of
all of them, and the clipping of the gradients by their global norm.

    python examples/train_encoder.py [--steps 20]

Texts are random token sequences of different lengths, laid back to back with int32 offsets; the query of a document is a noisy excerpt
of it, so that there is something to learn.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_29517_amd import autograd as A  # noqa: E402
from paper_2605_29517_amd import binding as M  # noqa: E402
from paper_2605_29517_amd.rope import rope_frequencies  # noqa: E402

VOCAB, WIDTH, HEADS, KV_HEADS, D, OUT = 1000, 256, 4, 2, 64, 128
TAU = 0.05


def parameters(seed=0, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def matrix(rows, cols):
        return (torch.randn(rows, cols, generator=g, device=device) / cols ** 0.5).requires_grad_()

    return {"tokens": torch.randn(VOCAB, WIDTH, generator=g, device=device).requires_grad_(), "qkv": matrix((HEADS + 2 * KV_HEADS) * D, WIDTH),
            "mix": matrix(WIDTH, HEADS * D), "out": matrix(OUT, WIDTH)}


def encode(p, tokens, offsets, freqs):
    """Token embeddings [T, OUT], unit rows, of packed texts: one layer in which every token of a text sees every other one."""
    x = p["tokens"][tokens]
    qkv = (x.bfloat16() @ p["qkv"].bfloat16().t()).view(-1, HEADS + 2 * KV_HEADS, D)
    qk = A.rope(qkv[:, :HEADS + KV_HEADS], freqs, offsets=offsets)  # queries and keys in one call
    o = A.attention(qk[:, :HEADS], qk[:, HEADS:], qkv[:, HEADS + KV_HEADS:], offsets, causal=False)
    x = x + (o.reshape(-1, HEADS * D) @ p["mix"].bfloat16().t()).float()
    return torch.nn.functional.normalize(x @ p["out"].t(), dim=-1).half()


def batch(seed, n=16, l_q=16, lo=20, hi=90, device="cuda"):
    """n documents of lo to hi tokens, packed, and a query of l_q tokens to each: tokens of the document, three quarters of them replaced."""
    g = torch.Generator().manual_seed(seed)
    lengths = torch.randint(lo, hi + 1, (n,), generator=g)
    offsets = torch.zeros(n + 1, dtype=torch.int32)
    offsets[1:] = torch.cumsum(lengths, 0)
    docs = torch.randint(0, VOCAB, (int(offsets[-1]),), generator=g)
    queries = torch.stack([docs[int(a) + torch.randint(0, int(l), (l_q,), generator=g)] for a, l in zip(offsets, lengths)])
    noise = torch.rand(n, l_q, generator=g) < 0.75
    queries[noise] = torch.randint(0, VOCAB, (int(noise.sum()),), generator=g)
    q_offsets = torch.arange(0, n * l_q + 1, l_q, dtype=torch.int32)
    return docs.to(device), offsets.to(device), queries.flatten().to(device), q_offsets.to(device)


def step(p, data, freqs, lr=0.2, max_norm=1.0):
    """One step of gradient descent: loss and global norm of the gradients before they were clipped, both on the GPU."""
    docs, offsets, queries, q_offsets = data
    n = offsets.numel() - 1
    Q = encode(p, queries, q_offsets, freqs).view(n, -1, OUT)
    D = encode(p, docs, offsets, freqs)
    scores = A.maxsim(Q, D, offsets)
    loss = torch.nn.functional.cross_entropy(scores / (TAU * Q.shape[1]), torch.arange(n, device=docs.device))
    grads = torch.autograd.grad(loss, list(p.values()))
    norm = M.maxsim_clip_grad_norm(grads, max_norm)  # in place
    with torch.no_grad():
        for w, g in zip(p.values(), grads):
            w -= lr * g
    return loss.detach(), norm


def train(steps, seed=0):
    p = parameters(seed)
    freqs, _ = rope_frequencies(D, device="cuda")
    return [tuple(float(x) for x in step(p, batch(seed + 1 + i % 4), freqs)) for i in range(steps)]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    for i, (loss, norm) in enumerate(train(ap.parse_args().steps)):
        print("step %3d  loss %.4f  gradient norm %.3f" % (i, loss, norm), flush=True)
