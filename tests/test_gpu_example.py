"""The attention example at a small size: compressed projections, norms, the
cache and attention as a program uses them, prompts and a replayed graph.  P and
the output are rounded to 8 significant bits each: 2^-8 of the result at most,
so 2^-7 in the norm."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_attention_block():
    spec = importlib.util.spec_from_file_location(
        "attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    errors = m.run(hidden=256, heads=4, kv_heads=2, prompts=(20, 70, 3), steps=5)
    assert len(errors) == 3 and max(errors) <= 2.0 ** -7, errors
