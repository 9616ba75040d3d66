"""The example runs the language-model operators and the search together; its results are what they are for."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_retrieval_decode():
    spec = importlib.util.spec_from_file_location("retrieval_decode", os.path.join(ROOT, "examples", "retrieval_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    got = m.main(states=60_000, batch=64, steps=20)
    assert got["losses"][-1] < got["losses"][0]      # the gradient goes down
    assert got["mixed"] < got["own"]                 # the neighbours know more of what followed
    assert got["right"] > 0.5
