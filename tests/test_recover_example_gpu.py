"""The recovery example end to end: the grouped products with their gradients, AdamW and the 8-bit products in one run."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_recovery_lowers_the_error_and_serves_in_8_bits():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recover_experts.py")
    spec = importlib.util.spec_from_file_location("recover_experts", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    before, after, rounding = example.run(d=256, E=8, I=384, T=512, steps=30)
    # training goes down; two roundings to 127 steps of a row and of a channel each add about a percent of the norm
    assert 0 < after < before
    assert 0 < rounding < 0.05
