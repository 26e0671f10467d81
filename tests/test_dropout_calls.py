"""How far a step advances the generator's offset: masks belong to offset + call."""
import itertools

import numpy as np

from tests import linear_reference as ref


def masks(offset, calls):
    return [ref.multiplier(16, 40, 0.4, 5, offset, c) for c in range(calls)]


def test_a_step_advances_by_its_calls():
    every = [m for step in range(3) for m in masks(100 + 4 * step, 4)]
    assert not any(np.array_equal(a, b) for a, b in itertools.combinations(every, 2))


def test_less_repeats_a_mask():
    assert np.array_equal(masks(100, 4)[1], masks(101, 4)[0])
