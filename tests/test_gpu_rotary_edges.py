"""Rotary positions where they are easy to get wrong: fractions of a turn between two of the 32-bit units in which angles are taken."""
import math

import pytest
import torch

from tests.gpu_util import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


@pytest.fixture(scope="module")
def B():
    from paper_2301_12017_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_are_the_nearest_of_their_units(B, interleaved):
    """Turns of some 2^-32 a position: the sine of an angle that small is the angle, off by half a unit (2 pi 2^-33) and, as a bf16 number, by 2^-8 of itself.  (The fp32 steps
    round relatively there: 2^-22 of it.)"""
    per = [0xFFFFFFFF, 0x180000001, 0x7FFFFFFF, 0x80000001, 0x2FFFFFFFF, 2 ** 64 - 0xFFFFFFFF, 2 ** 64 - 0x7FFFFFFF, 2 ** 64 - 0x1C0000000]
    angles = B.RotaryAngles(torch.zeros(8), interleaved)
    angles.turns.copy_(torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in per], dtype=torch.int64))
    x = torch.zeros((3, 1, 16), dtype=torch.bfloat16)
    b, a = (slice(1, 16, 2), slice(0, 16, 2)) if interleaved else (slice(8, 16), slice(0, 8))
    x[..., b] = 1
    got = B.rotary(x.cuda(), torch.tensor([1, 2, 3], dtype=torch.int32).cuda(), angles).cpu().double()
    for i, p in enumerate((1, 2, 3)):
        turn = torch.tensor([((t * p + 2 ** 63) % 2 ** 64 - 2 ** 63) / 2.0 ** 64 for t in per], dtype=torch.float64)
        want = -torch.sin(2 * math.pi * turn)
        assert ((got[i, 0, a] - want).abs() <= 2 * math.pi * 2.0 ** -33 * (1 + 2.0 ** -7) + want.abs() * (2.0 ** -8 + 2.0 ** -20)).all(), (got[i, 0, a], want)
        assert (got[i, 0, b] == 1).all()
