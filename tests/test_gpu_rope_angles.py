"""Angles of occ_rope against exact ones: positions are whole, frequencies 64-bit fractions of a turn, and what occ.h promises
of their product is 2^-32 of a turn at every position.

Tolerance.  A pair (1, 0) turned by a gives (cos a, sin a) with no rounding but theirs, (0, 1) gives (-sin a, cos a).  The
sine and cosine are off by 2 ulp each, 2^-22 of their size, the angle's last bits add a product and a sum, 2^-24 each of a term that
is no larger: less than 2^-21 of the size, also where that is small, and next to nothing (2^-40) for the angle itself.  An angle that is
rounded to binary32, 2^-26 of a turn, is off by up to 9e-8 there, a thousand times that at a sine of 2^-9."""
import math

import numpy as np
import pytest
import torch

from gpu_common import DEV
from paper_2606_09200_amd import binding as occ

pytestmark = pytest.mark.gpu
TURN = 1 << 64


def cos_sin(phase):
    """cos and sin of 2 pi phase / 2^64 by its distance from the nearest quarter turn, exact in whole numbers."""
    quarter = (phase + (TURN >> 3)) // (TURN >> 2)
    a = 2 * math.pi * ((phase - quarter * (TURN >> 2)) / TURN)
    c, s = math.cos(a), math.sin(a)
    return ((c, s), (-s, c), (-c, -s), (s, -c))[quarter % 4]


def phases():
    rng = np.random.default_rng(5)
    out = [0, 1, -1, (1 << 39) - 1, 1 << 39, (1 << 39) + 1, TURN // 2, TURN // 2 - 1, TURN // 2 - (1 << 39), TURN // 4 + 1, 3 * TURN // 4 - 12345]
    for at in range(8):                      # around every eighth of a turn, near and far
        for bits in range(2, 61, 3):
            for sign in (-1, 1):
                out.append(at * (TURN // 8) + sign * (int(rng.integers(1 << (bits - 1), 1 << bits)) | 1))
    out += [int(rng.integers(0, 1 << 63)) * 2 + 1 for _ in range(200)]
    return out


def check(y, want):
    for got, w in zip(y.double().cpu().tolist(), want):
        for g, x in zip(got, w):
            assert abs(g - x) <= 2.0 ** -21 * abs(x) + 2.0 ** -40, (g, x)


@pytest.mark.parametrize("interleaved", [False, True])
def test_every_bit_of_the_angle(interleaved):
    """One position, frequencies of any 64 bits: a pair each."""
    all_phases = phases()
    all_phases += [0] * (-len(all_phases) % 256)
    for first in range(0, len(all_phases), 256):
        part = all_phases[first:first + 256]
        turns = torch.tensor([(p + TURN // 2) % TURN - TURN // 2 for p in part], dtype=torch.int64, device=DEV)
        x = torch.zeros((1, 2, 512), device=DEV)
        pairs = x.view(2, 256, 2) if interleaved else x.view(2, 2, 256).transpose(1, 2)
        pairs[0, :, 0], pairs[1, :, 1] = 1.0, 1.0
        occ.occ_rope(x, None, torch.tensor([1], dtype=torch.int32, device=DEV), turns, interleaved=interleaved)
        want = [cos_sin(p) for p in part]
        check(pairs[0], want)
        check(pairs[1], [(-s, c) for c, s in want])


@pytest.mark.parametrize("inverse", [False, True])
def test_far_positions(inverse):
    """The frequencies of a model at positions up to 2^31: what is left of millions of turns."""
    turns = occ.rope_turns(64, base=1e4)
    positions = [1, 2, 1000, 131071, 10 ** 6 + 3, 2 ** 24 + 1, 2 ** 30 - 1, 2 ** 31 - 1, -1, -77777, -2 ** 31]
    x = torch.zeros((len(positions), 1, 128), device=DEV)
    x[:, :, :64] = 1.0
    occ.occ_rope(x, None, torch.tensor(positions, dtype=torch.int32, device=DEV), turns, inverse=inverse)
    for r, p in enumerate(positions):
        want = [cos_sin(p * t * (-1 if inverse else 1)) for t in turns.tolist()]
        check(x[r, 0].view(2, 64).t(), want)
