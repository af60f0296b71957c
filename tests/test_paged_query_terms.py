"""How the paged kernel splits bf16 queries into three e5m2 terms over an 8-bit cache, emulated bit by bit: a row is scaled by the
power of two that brings its largest entry into [2^14, 2^15), rounded to fp16, and its top byte is taken off three times."""
import numpy as np
import pytest


def split(x):
    """The sum of the three terms of x (float32, |x| < 2^15)."""
    h, total = x.astype(np.float16), np.zeros(x.shape, np.float64)
    for _ in range(3):
        top = (h.view(np.uint16) & np.uint16(0xFF00)).view(np.float16)
        total += top.astype(np.float64)
        h = (h - top).astype(np.float16)
    return total


def bf16_binade(e):
    """All bf16 numbers of [2^e, 2^(e+1))."""
    return ((128 + np.arange(128)) * 2.0 ** (e - 7)).astype(np.float32)


@pytest.mark.parametrize("largest", [14, 14.99])
def test_entries_of_2_to_the_minus_23_of_the_largest_are_exact(largest):
    top = 2.0 ** 14 if largest == 14 else 32640.0          # the largest entry is at either end of its binade
    for e in range(14, -25, -1):
        x = bf16_binade(e)
        x = x[x <= top]
        wrong = np.abs(split(x) - x.astype(np.float64))
        if e >= -9:                                        # 2^-9 is 2^-23 of 2^14
            assert (wrong == 0).all(), e
        assert (wrong < 2.0 ** -30 * top).all(), e


def test_and_those_of_2_to_the_minus_24_are_not():
    x = bf16_binade(-10)
    assert (split(x) != x).sum() == 64


def test_rows_below_the_scaling_are_exact_all_the_same():
    """A row whose largest entry is below 2^-112 is scaled by 2^126: multiples of 2^-133 become multiples of 2^-7."""
    x = np.arange(1, 256, dtype=np.float32)
    for shift in range(-7, 7):                             # up to 2^14
        y = x * np.float32(2.0 ** shift)
        assert (split(y) == y).all(), shift
