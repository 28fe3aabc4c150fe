"""The example runs its operators together: the router learns under its mask, and the 4-bit layer serves from the
expert cache."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_router_and_4bit_experts():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "router_and_4bit_experts.py")
    spec = importlib.util.spec_from_file_location("example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(verbose=False)
    assert r["last_loss"] < 0.8 * r["first_loss"], r
    assert r["masked_load"] == 0 and r["fetches"] >= example.K and r["hits"] + r["fetches"] == 8 * example.K
    assert r["mx4_bytes"] * 3 < r["bf16_bytes"]
    assert 0.01 < r["mx4_error"] < 0.35, r  # weights and activations of 1 + 2 bits: an eighth to a quarter a value
