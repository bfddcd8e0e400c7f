"""How far numbers of pages of 8 bits are off, as the header states it, on the tests' own definition of insertion."""
import os
import re

import numpy as np
import pytest

from e4m3_util import Pages, VALUES
from paper_2406_10774_amd import binding as Q

D = 128
MOST = 61440.0
HALVES = np.arange(0x7c00, dtype=np.uint16).view(np.float16).astype(np.float64)     # magnitudes


def held_after(x, exponents):
    """What numbers x stand for, inserted into a page whose scale is 2^e for the first e and then grows to each of the others:
    before and after."""
    pages = Pages(np.zeros((1, 1, 2 + len(exponents), len(x) + 1), np.uint8), np.ones((1, 1)))

    def needs(e):                                                  # a channel that makes the scale 2^e
        return min(448.0 * 2.0 ** e, MOST) if e > -15 else 0.0

    pages.insert(0, 0, 0, np.concatenate([x, [needs(exponents[0])]])[None])
    first = VALUES[pages.codes[0, 0, 0, :-1]] * 2.0 ** exponents[0]
    for i, e in enumerate(exponents[1:]):
        pages.insert(0, 0, 1 + i, np.concatenate([0 * x, [needs(e)]])[None])
    assert pages.e[0, 0] == exponents[-1]
    return first, VALUES[pages.codes[0, 0, 0, :-1]] * 2.0 ** exponents[-1]


def numbers(e):
    return HALVES[HALVES <= min(448.0 * 2.0 ** e, MOST)]


LADDERS = ([[e] for e in range(-15, 9)] + [[e, e + 1] for e in range(-15, 8)] + [list(range(e, 9)) for e in range(-15, 7)] +
           [[-15, -13, -12, -8], [-10, -7, -4, -1], [-15, -14, 0, 1, 8], [-3, 0, 2, 3]])


@pytest.mark.parametrize("ladder", LADDERS, ids=lambda l: "_".join(map(str, l)))
def test_numbers_are_as_near_as_stated(ladder):
    """Inserted once: 2^-4 of the value or half a subnormal's step.  After growth: 2^-4 or less than a whole step of the last scale
    (rounding number i adds at most half a step of its scale, and each step is at most half of the next)."""
    x = numbers(ladder[0])
    first, last = held_after(x, ladder)
    assert (np.abs(first - x) <= np.maximum(2.0 ** -4 * x, 2.0 ** (ladder[0] - 10))).all()
    off = np.abs(last - x)
    assert ((off <= 2.0 ** -4 * x) | (off < 2.0 ** (ladder[-1] - 9))).all()


def test_growth_takes_more_than_half_a_step():
    """Why there are two statements: just under 1.5 steps of the last scale becomes two of the first, and then none."""
    x = np.array([0.0029278], np.float16).astype(np.float64)
    _, once = held_after(x, [1])
    _, grown = held_after(x, [0, 1])
    assert abs(once[0] - x[0]) <= 2.0 ** -9 and grown[0] == 0.0 and x[0] > 1.4 * 2.0 ** -9


def test_header_states_both():
    root = os.path.dirname(os.path.dirname(os.path.abspath(Q.__file__)))
    with open(os.path.join(root, "include", "quest.h")) as f:
        text = re.sub(r"[\s*]+", " ", f.read())
    assert "off by at most 2^-4 of its value or 2^-10 2^e, whichever is more" in text
    assert "less than 2^-9 2^e" in text
