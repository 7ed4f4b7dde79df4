"""The router and an instance's KV blocks together: examples/routed_prefill.py."""

import importlib.util
import os

import pytest

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_routed_requests_are_prefilled_from_their_hit_and_decoded():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "routed_prefill.py")
    spec = importlib.util.spec_from_file_location("routed_prefill", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    s = example.run()
    assert s["requests"] > 20 and s["decoded"] == 4 * s["requests"]
    assert s["hit"] > s["tokens"] // 10  # later turns and samples find their prefix
    # Both sides start from the same bf16 projections (values of standard deviation 1).  Rounded on the way
    # to bf16 here and not there: rotated queries and keys (2^-8 each, so scores of magnitude up to 8 are off by
    # 2^-8 * sqrt(2 / 64) * 8 * 8 at most), the weights (2^-8) and the output (2^-8 of up to 4).
    assert s["worst"] < 0.1
