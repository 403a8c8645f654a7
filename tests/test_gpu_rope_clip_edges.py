"""maxsim_rope and maxsim_clip_grad_norm at the ends of their sizes and numbers."""
import math

import pytest
import torch

from paper_2605_29517_amd import binding as M

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_rope_of_more_tokens_than_one_grid_dimension_takes():
    """2^24 + 3 tokens of a width that leaves each a workgroup of its own."""
    tokens, d = (1 << 24) + 3, 514
    row = torch.randn(1, 1, d, generator=torch.Generator().manual_seed(1)).half().to(DEV)
    freqs = torch.full((d // 2,), 0.25, device=DEV)
    got = M.maxsim_rope(row.expand(tokens, 1, d), freqs)
    torch.cuda.synchronize()
    for at in (0, 1000, 1 << 22, (1 << 22) + 1, 1 << 23, tokens - 5):
        positions = torch.arange(at, at + 5, dtype=torch.int32, device=DEV)
        assert torch.equal(got[at:at + 5], M.maxsim_rope(row.expand(5, 1, d), freqs, positions=positions)), at


def test_clip_norms_beyond_fp32():
    """Gradients whose norm is beyond fp32, though each of them is not: the norm comes back as inf, the clipped gradients are as the formula has them."""
    for value, n in ((3e38, 5000), (1e38, 100), (3.4e38, 70_001)):
        g = [torch.full((n,), value, device=DEV), torch.full((3,), -value, device=DEV), torch.full((9,), 1.0, device=DEV)]
        want = [(t.double() / (float(torch.tensor(value)) * math.sqrt(n + 3))) for t in g]
        norm = M.maxsim_clip_grad_norm(g, 1.0)
        torch.cuda.synchronize()
        assert float(norm) == math.inf
        for t, w in zip(g, want):
            # the factor is an fp32 number of the size of its smallest normal ones: 2^-21 of it, and half the distance of the smallest results
            assert ((t.double() - w).abs() <= 2.0 ** -21 * w.abs() + 2.0 ** -149).all()
