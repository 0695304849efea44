"""The example runs the reading calls together: what it learns falls to its lists, and serving gives what training gave."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_the_example_learns_and_answers_from_its_lists():
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer.py")
    spec = importlib.util.spec_from_file_location("answer", at)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.main(steps=25, questions=16)
    assert got["losses"][-1] < 0.5 * got["losses"][0]
    assert got["in_list"]
    # two parts rounded to bfloat16 (2^-9 each of their share) and a key's weight 2^-8 off, against one sum: below 2^-6
    assert got["off_by"] < 2.0 ** -6
