"""Sines of rotary positions in 32 bits, near where they vanish: what the angle is off by is all that is left of them there."""
import math

import pytest
import torch

from paper_2201_12023_amd import blocks as B
from tests.layer_cases import D, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("quarter", [1, 2, 3, 5, 6, 7, 403, 4002])
def test_angles_keep_more_than_32_bits(quarter, interleaved):
    """Angles 1e-6 to 1e-2 of a turn beside quarter turns.  The angle, p f, and its part of a turn are off by 2^-52 each of up to 1001 turns, 2^-39 of a radian; a sine and a cosine
    by 4 units of 2^-24 of themselves."""
    g, rows, half = gen(61), 50, 8
    pos = torch.arange(1, rows + 1, device="cuda")
    delta = 10.0 ** (-6 + 4 * torch.rand(half, dtype=D, device="cuda", generator=g))
    for row in (0, 3, 49):
        p = int(pos[row])
        f = 2 * math.pi * (quarter / 4.0 + delta) / p
        x = torch.zeros(rows, 1, 2 * half, device="cuda")
        (x[..., 0::2] if interleaved else x[..., :half]).fill_(1.0)
        angle = p * f
        for call, sign in ((B.alpa_rotary_forward, 1.0), (B.alpa_rotary_backward, -1.0)):
            y = call(x, pos, f, interleaved)[row, 0].to(D)
            cos, sin = (y[0::2], y[1::2]) if interleaved else (y[:half], y[half:])
            for got, ref in ((cos, torch.cos(angle)), (sin, sign * torch.sin(angle))):
                assert float(((got - ref).abs() - 4 * 2.0 ** -24 * ref.abs()).max()) <= 2.0 ** -38
