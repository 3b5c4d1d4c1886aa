"""Pins of the oracle's append to blocks whose scale is no power of two, on the CPU."""
import numpy as np
import pytest

from oracle import history_operators as ho


@pytest.mark.parametrize("scale,row,after,older", [(3.0, 96.0, 4.0, 30.0), (3.0, 4000.0, 16.0, 30.0), (1.5, 1.0, 2.0, 15.0), (4.0, 96.0, 4.0, 40.0),
                                                   (2.0 ** -110, 0.0, 2.0 ** -100, 10 * 2.0 ** -110), (0.0, 0.0, 2.0 ** -100, 0.0)])
def test_older_rows_stand_for_what_they_did(scale, row, after, older):
    cache, scales = np.full((1, 1, 64, 4), 10.0), np.full((1, 1, 1), scale)
    ho.append(cache, scales, np.full((1, 1, 1, 4), row), [2])
    assert scales[0, 0, 0] == after
    assert abs(cache[0, 0, 0, 0] * after - older) <= max(2.0 ** -4 * older, 2.0 ** -10 * after)
    assert abs(cache[0, 0, 2, 0] * after - row) <= 2.0 ** -4 * row


def test_smallest_power_at_or_above():
    for s, e in ((0.0, -100), (2.0 ** -149, -100), (2.0 ** -100, -100), (1.0, 0), (1.0000001, 1), (3.0, 2), (2.0 ** 120, 120), (1.5 * 2.0 ** 123, 120)):
        assert ho.power_at_or_above(s) == e
