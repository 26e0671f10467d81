"""Every launch of a layer that the card's memory could hold has fewer than 2^32 threads, however tall the layer (plans only)."""
import re

import pytest

from paper_2512_06989_amd import mhffn
from tests.test_gpu_linear_plans import plan

MEMORY = 280e9
THREADS = {"bf16": {"256x256": 512, "256x128": 512, "128x128": 512, "64x128": 256, "64x64": 256}, "f32": {"128x128": 256, "64x64": 256}}


def threads(dt, text, M, N):
    m = re.match(r"(\d+)x(\d+) splits=(\d+)", text)
    a, b, splits = (int(v) for v in m.groups())
    return -(-M // a) * -(-N // b) * splits * THREADS[dt]["%dx%d" % (a, b)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1 << 25, 200000000, 1 << 28])
def test_tall_layers(M, dt):
    held = 0
    for a in (1, 7, 32, 64, 100, 256):
        for b in (1, 33, 64, 65, 129, 193, 257, 320, 321, 384, 450, 512, 1000, 1025, 2048, 2304):
            if M * (a + b) * (2 if dt == "bf16" else 4) > MEMORY:
                continue
            held += 1
            text = plan(mhffn.OP_LINEAR_FORWARD, dt, (M, a, b))
            if "few rows" not in text:
                assert threads(dt, re.search(r"\d+x\d+ splits=\d+$", text).group(0), M, b) < 2 ** 32, (a, b, text)
            text = plan(mhffn.OP_LINEAR_BACKWARD, dt, (M, b, a))
            dX, dW = re.search(r"dX (.*?)(?:; dW| with dW) (.*)", text).groups()
            both = [threads(dt, dX, M, b) if "few" not in dX else 0, threads(dt, dW, b, a)]
            assert (sum(both) if " with dW" in text else max(both)) < 2 ** 32, (b, a, text)
    assert held > 20
