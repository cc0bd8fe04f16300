"""The example that runs router, compression, aggregation, norm and AdamW
together: it learns, with 32- and with 8-bit moments."""
import importlib.util
import math
import os

import pytest

from _gpu_common import log

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("moe_router", os.path.join(ROOT, "examples", "moe_router.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("bits", [32, 8])
def test_learns(example, bits):
    history = example.train(steps=80, state_bits=bits, log=log)
    assert all(math.isfinite(x) for row in history for x in row)
    first, last = history[0], history[-1]
    assert last[0] < 0.5 * first[0], "the task loss halves at least"
    assert last[1] < 1.5, "the experts stay in use"
