"""examples/serve_samples.py runs, and what it checks holds."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_serve_samples():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_samples.py")
    spec = importlib.util.spec_from_file_location("serve_samples", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main()
    # FP16 weights and an FP16 result, 2^-11 each of values that are at most a few times the largest result: 150 to 300 tokens of random values average to a tenth
    assert r["worst"] < 2.0 ** -7
    # INT8 with one scale to a page: half a step of 1/127 of the page's largest value, which is no more than the largest of all, and FP16
    assert r["loss"] < 0.5 / 127 + 2.0 ** -10
    # one sample ended, but the others share its prompt's blocks
    assert 0 < r["used_after"] < r["used_before"] and r["live_at_end"] == 0
