"""The example that runs the operators for learned inputs and large answers together learns, and its 8-bit table answers as its fp32 one."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_learns_and_answers_alike_from_eight_bits():
    spec = importlib.util.spec_from_file_location("learned_vertices", os.path.join(ROOT, "examples", "learned_vertices.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main(120, say=lambda text: print(text, flush=True))
    # the teacher's distribution has a floor that the student cannot get under; half of the way down is far more than noise
    assert r["last"] < 0.6 * r["first"]
    # 47 classes: guessing is right in 2 of 100
    assert r["fp32"]["right"] > 0.8 and r["fp32"]["among_three"] >= r["fp32"]["right"]
    # e4m3 is off by at most 2^-4 a value, independently: over 64 values and a few neighbours' mean about 1 % of a logit's spread
    assert abs(r["8 bits"]["logprob"] - r["fp32"]["logprob"]) < 0.05 and abs(r["8 bits"]["right"] - r["fp32"]["right"]) < 0.03
