"""8-bit floats of a paged cache, from their definition in 64 bits."""
import torch

import paper_2012_00596_amd as npas

BLOCK = 32
LIMITS = {npas.BF16: (-110, 120), npas.F16: (-15, 8)}   # exponents of a scale
GRID = torch.tensor([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:119],
                    dtype=torch.float64)                  # the numbers 0 .. 448 by their codes 0 .. 126


def dequantise(codes, scales):
    """codes uint8 [..., D], scales uint8 [..., ceil(D / 32)]: the values in 64 bits."""
    c = codes.long()
    v = torch.cat([GRID, torch.tensor([float("nan")], dtype=torch.float64)])[c & 127]
    unit = torch.where(scales == 255, float("nan"), torch.exp2(scales.double() - 127)).repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]
    return torch.where(c >= 128, -v, v) * unit


def exponents(x, dt):
    """The exponents of x's blocks (64 bits, last axis a head), before the limits; the largest magnitudes."""
    D = x.shape[-1]
    top = torch.nn.functional.pad(x, (0, -D % BLOCK)).unflatten(-1, (-1, BLOCK)).abs().amax(-1)
    e = torch.frexp(top)[1] - 9                            # top = m 2^(e + 9), m in [1/2, 1): at most 448 2^e = 7/8 2^(e + 9) where m is
    return e + (torch.frexp(top)[0] > 0.875), top


def quantise(x, dt):
    """(codes, scale bytes) of x (64 bits, finite or not)."""
    D, (least, most) = x.shape[-1], LIMITS[dt]
    bad = ~torch.isfinite(torch.nn.functional.pad(x, (0, -D % BLOCK)).unflatten(-1, (-1, BLOCK))).all(-1)
    e, top = exponents(torch.where(torch.isfinite(x), x, 0.0), dt)
    e = torch.where(top == 0, least, e).clamp(least, most)
    unit = torch.exp2(e.double()).repeat_interleave(BLOCK, -1)[..., :D]
    cap = torch.where(e == most, 240.0, 448.0).double().repeat_interleave(BLOCK, -1)[..., :D]
    r = torch.minimum((torch.nan_to_num(x) / unit).abs(), cap)
    mids = (GRID[1:] + GRID[:-1]) / 2
    code = torch.searchsorted(mids, r)                     # the lower one of a tie
    tie = r == mids[code.clamp(max=125)]
    code = code + (tie & (code % 2 == 1) & (code < 126)).long()
    code = code | (torch.signbit(x).long() << 7)
    wide = bad.repeat_interleave(BLOCK, -1)[..., :D]
    return torch.where(wide, 127, code).to(torch.uint8), torch.where(bad, 255, e + 127).to(torch.uint8)
