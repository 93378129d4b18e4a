"""The example that trains a student of residual blocks from a graph network's largest logits, in each element type."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("type_", ["f32", "bf16", "f16"])
def test_student_learns_from_the_teacher(type_):
    spec = importlib.util.spec_from_file_location("distill_student", os.path.join(ROOT, "examples", "distill_student.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    lines = []
    first, last, agree = m.train(type_, blocks=2, width=64, steps=120, say=lines.append)
    assert last < 0.5 * first, (first, last)
    assert agree > 0.6, agree                      # eight classes; a guess agrees on an eighth
    assert any("vertex 0 alone" in x for x in lines)
