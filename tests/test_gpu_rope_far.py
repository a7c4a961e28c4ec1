"""Rotary angles at the far ends of frequencies and positions, against exact arithmetic.

A frequency becomes a whole number of 2^-64 turns per position, cut and rounded by at most 1.5 of them, so position p is off
by |p| 1.5 2^-64 turns.  Cosine and sine of the part of a turn: E, as derived in test_gpu_rope.py; one rounding for the
factor."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
from paper_2606_07571_b200 import binding

pytestmark = pytest.mark.gpu
E = 1.5e-7


@pytest.fixture(scope="module")
def bc():
    entry.build()
    return binding.BiCache(1, 2, 1, 128, 8, torch.bfloat16, 16, 1)


def inverse_two_pi(bits=256):
    """1 / (2 pi) as a fraction: pi = 16 atan(1/5) - 4 atan(1/239), alternating series in integers."""
    one = 1 << (bits + 16)

    def atan(x):
        term = total = one // x
        n, sign = 1, -1
        while term:
            term //= x * x
            n += 2
            total += sign * (term // n)
            sign = -sign
        return total
    return Fraction(one, 2 * (16 * atan(5) - 4 * atan(239)))


def exact(positions, freq):
    inv = inverse_two_pi()
    out = np.empty((len(positions), len(freq), 2))
    for i, f in enumerate(freq):
        turn = Fraction(float(f)) * inv
        for r, p in enumerate(positions):
            part = float((turn * int(p) + Fraction(1, 2)) % 1 - Fraction(1, 2))
            out[r, i] = np.cos(2 * np.pi * part), np.sin(2 * np.pi * part)
    return out


FREQ = np.concatenate([10000.0 ** (-np.arange(0, 64, 3) / 64), [2.0 ** 20, 1e5 / 3, 6.25, 0.0, 1e-9, 1e-18]])


@pytest.mark.parametrize("sign", [1, -1])
def test_far_int32_positions(bc, sign):
    pos = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, 1 << 30, 1 << 20, 1, 0]
    table = torch.empty((len(pos), len(FREQ), 2), device="cuda")
    bc.rope_table(sign * FREQ, table, positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    bound = E + 2.0 ** -24 + 2 * np.pi * 1.5 * 2.0 ** -33
    err = np.abs(table.double().cpu().numpy() - exact(pos, sign * FREQ))
    assert (err <= bound).all(), err.max()


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("position0", [2 ** 36 - 6, -2 ** 36, 2 ** 33 + 1, -2 ** 32 - 5])
def test_consecutive_positions_up_to_the_ends_of_their_range(bc, position0, sign):
    table = torch.empty((7, len(FREQ), 2), device="cuda")
    bc.rope_table(sign * FREQ, table, position0=position0)
    bound = E + 2.0 ** -24 + 2 * np.pi * 1.5 * 2.0 ** -28
    err = np.abs(table.double().cpu().numpy() - exact(range(position0, position0 + 7), sign * FREQ))
    assert (err <= bound).all(), err.max()
