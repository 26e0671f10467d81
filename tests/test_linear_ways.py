"""Which ways the GPU tests of the linear layer take at their sizes: every tile, shares of the contraction with each form that has
them, the shared launches, packed operands, and both kernels for few rows.  A cost that moves may not take one off the lists unseen."""
import re

import pytest

from paper_2512_06989_amd import mhffn
from tests.test_gpu_linear import SHAPES
from tests.test_gpu_linear_more_ways import SHAPES as MORE
from tests.test_gpu_linear_plans import BACKWARD, FORWARD, plan
from tests.test_gpu_linear_ragged_splits import SHAPES as RAGGED

TILES = ("256x256", "256x128", "128x128", "64x128", "64x64")
forward = {dt: [plan(mhffn.OP_LINEAR_FORWARD, dt, s) for d, s in FORWARD + [(t, s) for t in ("bf16", "f32") for s in SHAPES] if d == dt]
           for dt in ("bf16", "f32")}
backward = {dt: [plan(mhffn.OP_LINEAR_BACKWARD, dt, s) for d, s in BACKWARD + [(t, s) for t in ("bf16", "f32") for s in SHAPES + RAGGED] + [("bf16", s) for s in MORE] if d == dt]
            for dt in ("bf16", "f32")}


def some(ways, pattern):
    return any(re.search(pattern, w) for w in ways)


@pytest.mark.parametrize("tile", TILES)
def test_bf16_tiles(tile):
    assert some(forward["bf16"], r"(^|W |X )%s splits=1$" % tile)
    assert some(backward["bf16"], r"dX %s splits=1;" % tile)
    assert some(backward["bf16"], r"dX %s splits=([2-9]|1\d);" % tile)
    assert some(backward["bf16"], r"; dW %s splits=1$" % tile)
    assert some(backward["bf16"], r"; dW %s splits=([2-9]|1\d)$" % tile)


@pytest.mark.parametrize("way", [r"splits=[2-9]", r"^few rows$", r"few rows as they lie", r"packed W", r"packed X packed W"])
def test_bf16_forward(way):
    assert some(forward["bf16"], way), forward["bf16"]


@pytest.mark.parametrize("way", [r"with dW", r"packed X packed W dZ .*with dW",
                                 r"packed X packed W dZ .*; dW \S+ splits=([2-9]|1\d)", r"dX few rows"])
def test_bf16_backward(way):
    assert some(backward["bf16"], way), backward["bf16"]


@pytest.mark.parametrize("way", [r"^64x64 splits=1$", r"^64x64 splits=([2-9]|1\d)", r"^128x128 splits="])
def test_f32_forward(way):
    assert some(forward["f32"], way), forward["f32"]


@pytest.mark.parametrize("way", [r"splits=1 with dW \S+ splits=1$", r"dX \S+ splits=([2-9]|1\d) with dW", r"with dW \S+ splits=([2-9]|1\d)", r"; dW"])
def test_f32_backward(way):
    assert some(backward["f32"], way), backward["f32"]


def test_few_rows_of_both_kernels():
    """(weights in row form: up to 8 rows 16 columns a workgroup, above 32 x 32)"""
    assert "dX few rows" in plan(mhffn.OP_LINEAR_BACKWARD, "bf16", (3, 576, 6080)) and (3, 576, 6080) in MORE
    assert "dX few rows" in plan(mhffn.OP_LINEAR_BACKWARD, "bf16", (7000, 32, 64)) and (7000, 32, 64) in MORE
    assert {s[0] > 16 for d, s in FORWARD + [("bf16", s) for s in SHAPES] if d == "bf16" and plan(mhffn.OP_LINEAR_FORWARD, d, s) == "few rows"} == {True, False}
