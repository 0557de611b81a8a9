"""Rotary positions: what the angle itself may be off by."""
import math

import pytest
import torch

from paper_2609_36938_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_small_angles(interleaved):
    """x = (1, 0) turned by a phase of less than 2^-20 turns gives its sine: the phase is rounded to a multiple of 2^-32 turns, half a step or 2^-33 turns; angle, sine
    and product in fp32 2^-21 of it."""
    g = torch.Generator(device="cuda").manual_seed(1)
    freqs = torch.randint(0, 1 << 44, (64,), device="cuda", generator=g)
    freqs[0], freqs[1], freqs[2] = (1 << 32) - 1, (1 << 31) + 1, (1 << 31) - 1
    x = torch.zeros((1, 1, 128), device="cuda")
    first, second = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, 64), slice(64, None))
    x[..., first] = 1.0
    for pos in (1, 3):
        y = B.janus_rope(x, torch.tensor([pos], device="cuda"), freqs, interleaved=interleaved)
        want = torch.sin(freqs.double() * pos * 2.0 ** -64 * 2 * math.pi)
        err = (y[0, 0, second].double() - want).abs()
        assert (err <= 2 * math.pi * 2.0 ** -33 + 2.0 ** -21 * want).all(), float(err.max())
        assert ((y[0, 0, first].double() - 1.0).abs() <= 2.0 ** -21).all()
