"""The 64-bit forms of the 4-bit format against its definition, value by value."""
import math

import torch

from quant_util import GRID, quantised4, widened4
from serve_util import F64


def test_every_code_comes_back():
    codes = torch.arange(256, dtype=torch.uint8).view(16, 16)
    for e in (2, 100, 127, 200, 252):
        exps = torch.full((16, 1), e, dtype=torch.uint8)
        x = widened4(codes, exps)
        assert x[0, 2] == GRID[1] * 2.0 ** (e - 127) and x[0, 1] == 0 and x[15, 31] == -6 * 2.0 ** (e - 127)
        back = widened4(*quantised4(x))
        assert torch.equal(back, x)


def test_nearest_and_even():
    for value, want in ((0.25, 0), (0.2500001, 0.5), (0.75, 1), (1.25, 1), (1.26, 1.5), (1.75, 2), (2.5, 2), (3.5, 4), (5.0, 4), (5.0001, 6), (6.0, 6)):
        x = torch.zeros(64, dtype=F64)
        x[0], x[5], x[40] = 6.0, -value, value
        y = widened4(*quantised4(x))
        assert y[5] == -want
        # by itself a group takes the smallest power of two that holds it
        e = math.ceil(math.log2(value / 6.0))
        assert (y[40] / 2.0 ** e) in GRID and abs(y[40] - value) <= 2.0 ** e
    codes, exps = quantised4(torch.tensor([[1.0] * 31 + [float("nan")], [0.0] * 32, [-0.0] * 32], dtype=F64))
    assert exps[:, 0].tolist() == [255, 127, 127] and codes[0].tolist() == [0] * 16 and codes[2].tolist() == [0x88] * 16
    assert bool(torch.isnan(widened4(codes, exps)[0]).all())
