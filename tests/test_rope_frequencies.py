"""The scaling of angles by wavelength, pair by pair, where the original length is short, ordinary and very long (no GPU needed)."""
import math

import pytest
import torch

from paper_2605_29517_amd.rope import rope_frequencies


@pytest.mark.parametrize("original", [64, 2048, 8192, 65536, 131072, 1 << 20])
@pytest.mark.parametrize("rot,base,factor", [(64, 10000.0, 4.0), (128, 10000.0, 8.0), (128, 500000.0, 8.0), (32, 10000.0, 2.0)])
def test_parts_by_wavelength(rot, base, factor, original):
    """A pair that turns at least 32 times stays, one that turns at most once is interpolated in full, and one between them is neither; the share
    of interpolation grows by the same amount from pair to pair between the two pairs at which it starts and ends."""
    plain = rope_frequencies(rot, base=base)[0].double()
    freqs = rope_frequencies(rot, base=base, factor=factor, scaling="parts", original=original)[0].double()
    turns = original * plain / (2 * math.pi)
    share = (1 - freqs / plain) / (1 - 1 / factor)
    close = 1e-5  # angles are fp32 numbers
    assert (share[turns >= 32].abs() < close).all()
    assert ((share[turns <= 1] - 1).abs() < close).all()
    # the pairs between: 0 at the last pair that turns 32 times or more (the first pair where none does), 1 at the first one that turns once or less
    pair = torch.arange(rot // 2, dtype=torch.float64)
    at = lambda n: rot / 2 * math.log(original / (2 * math.pi * n)) / math.log(base)  # noqa: E731  (the pair that turns n times, a fraction)
    first, last = max(math.floor(at(32)), 0), math.ceil(at(1))
    if last > first:
        assert ((share - ((pair - first) / (last - first)).clamp(0, 1)).abs() < close).all()
    between = (turns < 31) & (turns > 1.1) & (pair > first)
    assert (share[between] < 1 - close).all() and (share[between] > 0).all()
