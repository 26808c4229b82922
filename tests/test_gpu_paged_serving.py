"""The serving example end to end: prompts by chunks, decode steps, and the contiguous read of what the
cache then holds (needs a GB300)."""
import importlib.util
import os

import pytest

from paper_2602_07160_gb300 import build, fem

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    build.build()
    fem.load()
    spec = importlib.util.spec_from_file_location("paged_serving", os.path.join(ROOT, "examples", "paged_serving.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_paged_serving(example, fmt):
    worst, lens = example.serve([5, 300, 64, 129], tokens=4, fmt=fmt, width=128, q_heads=8, heads=2, d=64, page=32, chunk=100)
    assert lens == [9, 304, 68, 133]
    # bf16 outputs of values of order one: their rounding and the bank's, each 2^-8 of a value up to about 4
    assert worst <= 2.0 ** -8 * 8
