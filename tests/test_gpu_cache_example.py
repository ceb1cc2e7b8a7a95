"""The example that runs append and attention together, on a small video."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_cached_blocks():
    spec = importlib.util.spec_from_file_location("cached_blocks", os.path.join(ROOT, "examples", "cached_blocks.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.main(["--blocks", "3", "--tokens", "200", "--heads", "4", "--steps", "2"])
    # A held value is off by up to half a step, a thirtieth of its group's range: about a tenth of the values' spread, in keys and in
    # values; flat softmax averages that of the values, and a softmax output of random values is as small as its average
    assert 0.0 < got["worst"] < 0.35
    assert got["wide"] > 3.4 * got["held"]
    assert torch.isfinite(got["last"]).all()
