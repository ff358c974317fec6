"""The example of a token model with experts: it learns, in every storage type."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_it_learns(kind):
    spec = importlib.util.spec_from_file_location("train_experts", os.path.join(ROOT, "examples", "train_experts.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, right = example.main(steps=120, kind=kind, quiet=True)
    # (512 tokens, a table that is its own output: the first loss is above log 512 = 6.2)
    assert first > 6.0 and last < 0.5 and right > 0.9, (first, last, right)
