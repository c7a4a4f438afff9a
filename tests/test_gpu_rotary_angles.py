"""Sines and cosines of rotary positions next to multiples of a quarter turn."""
import math

import pytest
import torch

import streams_reference as ref
from paper_2608_26965_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("adjacent", [True, False])
@pytest.mark.parametrize("inverse", [False, True])
def test_small_sines_and_cosines_are_accurate_too(adjacent, inverse):
    """Of (1, 0) the rotation gives cosine and sine alone.  The phase is exact to 2^-64 of a turn per step; its remainder from the
    nearest quarter turn is rounded once (u of it, as much of the sine), sine and cosine of that are off by 2 ulp (4 u): 6 u of the value.
    The 64-bit angle here, up to 70 radians, is off by 2^-53 70 < 1e-14, twice that with 2 pi."""
    off = [0.0, 1e-7, -3e-6, 1e-4, -2e-3, 0.05, 0.7, 1e-9]
    freqs = [math.pi / 2 + x for x in off] + [math.pi / 4 + x for x in off] + [math.pi + x for x in off] + [1e-3 * (1 + i) for i in range(8)]
    rot = binding.Rotary(64, [32], frequencies=freqs, adjacent=adjacent)
    n = 41
    pos = (torch.arange(n, device=DEV, dtype=torch.int32) - 20).view(1, n, 1)
    x = torch.zeros((1, 1, n, 64), device=DEV)
    if adjacent:
        x[..., 0::2] = 1.0
    else:
        x[..., :32] = 1.0
    y = binding.rotary_axes(rot, x, None, pos, inverse=inverse)[0][0, 0]
    cos, sin = (y[:, 0::2], y[:, 1::2]) if adjacent else (y[:, :32], y[:, 32:])
    t = pos.view(n, 1).double() * torch.tensor(freqs, dtype=torch.float64, device=DEV) * (-1.0 if inverse else 1.0)
    for got, want, what in ((cos, torch.cos(t), "cosine"), (sin, torch.sin(t), "sine")):
        ref.check(got, want, 6 * ref.U32 * want.abs() + 3e-14, what)
