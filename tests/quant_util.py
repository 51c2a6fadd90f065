"""Plain 64-bit forms of what is held in 4 bits: e2m1 codes, two to a byte, with a power of two for every 32 entries."""
import torch

from serve_util import F64

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F64)


def quantised4(x):
    """codes (uint8 [.., n/2]) and biased exponents (uint8 [.., n/32]) of x [.., n], from the definition: the nearest value of the grid, of two equally near ones that
    with the even code; the smallest exponent, 2 or more, that keeps the largest within 6; 127 for zeros; 255 where one is not finite."""
    x = x.to(F64).unflatten(-1, (-1, 32))
    bad = ~torch.isfinite(x).all(-1)
    x = torch.where(bad[..., None], torch.zeros_like(x), x)
    top = x.abs().amax(-1)
    e = torch.full(top.shape, 254, dtype=torch.int64)
    for b in range(253, 1, -1):
        e = torch.where(top <= 6.0 * 2.0 ** (b - 127), torch.full_like(e, b), e)
    assert bool((e < 254).all())
    e = torch.where(top == 0, torch.full_like(e, 127), e)
    a = torch.ldexp(x.abs(), 127 - e[..., None])
    off = (a[..., None] - GRID).abs()
    near = off == off.amin(-1, keepdim=True)
    code = torch.arange(8)
    pick = torch.where(near, code + 100 * (code % 2), torch.full_like(code, 1000)).argmin(-1)
    code = pick + 8 * torch.signbit(x).to(torch.int64)
    code = torch.where(bad[..., None], torch.zeros_like(code), code).flatten(-2)
    e = torch.where(bad, torch.full_like(e, 255), e)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), e.to(torch.uint8)


def widened4(codes, exps):
    """Their values [.., n] in 64 bits."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    x = GRID[c % 8] * torch.where(c >= 8, -1.0, 1.0)
    scale = torch.where(exps == 255, torch.full(exps.shape, float("nan"), dtype=F64), torch.ldexp(torch.ones(exps.shape, dtype=F64), exps.int() - 127))
    return (x.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


# Layers whose contraction is more than twice what the rings of their tile hold (tile; rows, contraction, columns): whole blocks of 128, and half a one at the end.
WRAPPED = [((16, 16), 3, 8320, 64), ((16, 16), 4, 8384, 128), ((16, 16), 13, 6272, 64), ((16, 16), 5, 6336, 192),
           ((16, 32), 13, 4224, 4160), ((16, 32), 5, 4288, 4224),
           ((16, 64), 20, 4224, 4160), ((16, 64), 29, 4288, 4224),
           ((32, 64), 33, 1664, 5504), ((32, 64), 47, 1728, 5504),
           ((64, 64), 65, 1920, 5504), ((64, 64), 100, 1984, 5568),
           ((64, 128), 129, 1664, 5504), ((64, 128), 150, 1728, 5568),
           ((64, 256), 257, 1152, 6592), ((64, 256), 300, 1216, 6656),
           ((128, 256), 513, 896, 7232), ((128, 256), 600, 960, 7296)]
