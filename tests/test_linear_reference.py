"""Pins of the linear layer's reference (CPU): the generator against its published known answers,
the mask's layout by hand, gradients against differences."""
import numpy as np
import pytest
import torch

from tests import linear_reference as ref


@pytest.mark.parametrize("counter,key,words", [
    (0, 0, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
    (2 ** 128 - 1, 2 ** 64 - 1, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
    (0x0370734413198a2e85a308d3243f6a88, 0x299f31d0a4093822, "d16cfe09 94fdcceb 5001e420 24126ea1"),
])
def test_known_answers_of_the_generator(counter, key, words):
    got = ref.philox([counter % 2 ** 64], key, counter >> 64)[0]
    assert " ".join("%08x" % w for w in got) == words


def test_layout_of_the_mask():
    seed, offset, call, rows, cols, p = 99, 2 ** 64 - 2, 5, 3, 21, 0.3    # (offset + call wraps)
    m = ref.multiplier(rows, cols, p, seed, offset, call)
    for i in range(rows):
        for j in range(cols):
            w = int(ref.philox([i * 3 + j // 8], seed, 3)[0][j % 8 // 2])
            half = (w >> 16) if j % 2 else (w & 0xFFFF)
            assert m[i, j] == (65536 / (65536 - 19661) if half >= 19661 else 0.0)
    assert np.array_equal(ref.multiplier(1, cols, p, seed, offset, call, first_row=2), m[2:])


def test_kept_share():
    for p in (0.1, 0.5, 0.9):
        kept = np.mean(ref.multiplier(1000, 1000, p, 7, 0, 0) != 0)
        assert abs(kept - (1 - p)) < 5 * 0.5 / 1000      # five standard deviations
    assert np.all(ref.multiplier(9, 9, 1.0, 7, 0, 0) == 0) and np.all(ref.multiplier(9, 9, 2.0 ** -18, 7, 0, 0) == 1)


@pytest.mark.parametrize("name", ref.ACTS)
def test_gradients_against_differences(name):
    r = np.random.default_rng(3)
    X, W, b, R = r.normal(size=(5, 7)), r.normal(size=(7, 9)), r.normal(size=9), r.normal(size=(5, 9))
    dY, mult = r.normal(size=(5, 9)), ref.multiplier(5, 9, 0.3, 1, 2, 3)
    loss = lambda X, W, b: float(np.sum(dY * ref.forward(X, W, b, R, name, mult, torch.float32)[0]))  # noqa: E731
    Z = ref.forward(X, W, b, R, name, mult, torch.float32)[2]
    grads = ref.backward(X, W, Z, dY, name, mult, torch.float32)
    for key, t, k in (("dX", X, 0), ("dW", W, 1), ("dbias", b, 2)):
        for i in np.ndindex(t.shape):
            args = [[a.copy() for a in (X, W, b)] for _ in range(2)]
            args[0][k][i] += 1e-5
            args[1][k][i] -= 1e-5
            assert abs((loss(*args[0]) - loss(*args[1])) / 2e-5 - grads[key][0][i]) < 1e-6
