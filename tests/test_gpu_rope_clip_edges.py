"""maxsim_rope and maxsim_clip_grad_norm at the ends of their sizes and numbers."""
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
