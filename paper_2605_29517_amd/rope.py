"""The angles per position that maxsim_rope takes, with the usual scalings for contexts longer than the model was trained on."""
import math

import torch


def rope_frequencies(rot, base=10000.0, factor=1.0, scaling=None, original=4096, fast=32.0, slow=1.0, device=None):
    """(freqs, scale) for maxsim_rope: freqs fp32 [rot / 2], the angle per position of pair i, base^(-2 i / rot) where nothing is scaled, and
    the factor that goes with them (1 but for "parts").

    scaling, for contexts `factor` times as long as the `original` ones:
      None     as trained
      "linear" positions are interpolated: every angle is divided by factor
      "base"   the base grows by factor^(rot / (rot - 2)): the slowest pair is interpolated by factor, the fastest one stays
      "parts"  by wavelength, the method of "YaRN: Efficient Context Window Extension of Large Language Models" (Peng et al., 2023): pairs that turn
               at least `fast` times within the original length stay, those that turn at most `slow` times are interpolated, between them the
               angle goes over linearly (in the pair's number); cosines and sines are scaled by 0.1 ln(factor) + 1, which sharpens the softmax
               of the longer rows
    """
    if rot < 2 or rot % 2:
        raise ValueError("rot must be even and at least 2")
    if not factor >= 1.0:
        raise ValueError("factor must be at least 1")
    pair = torch.arange(0, rot, 2, dtype=torch.float64)
    scale = 1.0
    if scaling is None or factor == 1.0:
        freqs = base ** (-pair / rot)
    elif scaling == "linear":
        freqs = base ** (-pair / rot) / factor
    elif scaling == "base":
        if rot == 2:
            raise ValueError("a single pair has no base to scale")
        freqs = (base * factor ** (rot / (rot - 2))) ** (-pair / rot)
    elif scaling == "parts":
        freqs = base ** (-pair / rot)

        def number(turns):  # of the pair that turns so many times within the original length
            return rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))

        # (the end may lie past the last pair, which then is not interpolated in full; the bounds 0 and rot - 1 are the published ones)
        first, last = max(math.floor(number(fast)), 0), min(math.ceil(number(slow)), rot - 1)
        share = ((pair / 2 - first) / max(last - first, 1e-3)).clamp(0.0, 1.0)  # of the interpolated angle
        freqs = freqs * (1.0 - share) + freqs / factor * share
        scale = 0.1 * math.log(factor) + 1.0
    else:
        raise ValueError("scaling must be None, 'linear', 'base' or 'parts'")
    return freqs.to(torch.float32).to(device), scale
