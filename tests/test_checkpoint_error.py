"""How far a value of an 8-bit checkpoint is off, as include/vardrop.h states it, evaluated with the oracle (which the kernels equal byte for byte)."""
import numpy as np
import pytest

from oracle import feedforward as o

LEAST, MOST = 63.75 * 2.0 ** -126, 127.5 * 2.0 ** 121


def off(block):
    """Largest error of a block, over its largest magnitude."""
    x = np.zeros((1, 32))
    x[0, :len(block)] = np.float32(block)
    return float(np.abs(o.through_8_bits(x) - x).max()), float(np.abs(x).max())


@pytest.mark.parametrize("e", [-120, -30, 0, 7, 60, 121])
def test_half_a_step_between_the_ends(e):
    """At most 1/127.5 of the block's largest; just above 63.75 steps a little more than 2^-7 of it."""
    worst = 0.0
    for most in np.linspace(63.75, 127.4999, 300):
        for part in (0.5, 1.5, 20.5, 31.499, 62.5):
            error, largest = off([most * 2.0 ** e, part * 2.0 ** e, -part * 2.0 ** e])
            if LEAST <= largest < MOST:
                assert error <= largest / 127.5 * (1 + 2.0 ** -23)
                worst = max(worst, error / largest)
    assert worst > 2.0 ** -7


def test_below_the_least_step():
    """A step of 2^-126: off by at most half of it, which may be all of the value."""
    for most in (63.7, 5.0, 0.5, 0.0625):
        error, largest = off([most * 2.0 ** -126, 0.3 * 2.0 ** -126])
        assert largest < LEAST and error <= 2.0 ** -127
    assert off([2.0 ** -130]) == (2.0 ** -130, 2.0 ** -130)


def test_past_the_largest_step():
    """Magnitudes from 127.5 * 2^121 on count as 127 * 2^121: off by less than a step."""
    error, largest = off([np.finfo(np.float32).max])
    assert largest >= MOST and 2.0 ** 120 < error < 2.0 ** 121
