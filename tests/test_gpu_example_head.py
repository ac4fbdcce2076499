"""The example of the output head, trained, quantised and served through the public calls: it learns, and its 4-bit form answers as it learnt."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def test_example_learns_and_serves(repo_root):
    spec = importlib.util.spec_from_file_location("output_head_example", os.path.join(repo_root, "examples", "output_head.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    before, after, agree = example.main(tokens=256, hidden=128, vocab=3001, steps=40, quiet=True)
    assert abs(before - math.log(3001)) < 0.5      # knows nothing
    assert after < before / 2 and agree > 0.9
