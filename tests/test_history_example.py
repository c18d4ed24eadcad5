"""What examples/user_histories.py compares with: a wrong stage has to show.  No device."""
import importlib.util
import os

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("user_histories", os.path.join(HERE, "..", "examples", "user_histories.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_a_result_that_is_not_finite_shows(example):
    want = torch.tensor([1.0, -4.0])
    assert example.off_by(want.bfloat16(), want) == 0.0
    assert example.off_by(torch.tensor([2.0, -4.0]), want) == 0.25
    for bad in (float("nan"), float("inf")):
        with pytest.raises(ArithmeticError):
            example.off_by(torch.tensor([bad, -4.0]), want)
        with pytest.raises(ArithmeticError):
            example.off_by(want, torch.tensor([1.0, bad]))
    with pytest.raises(ArithmeticError):       # another shape would be compared by broadcasting
        example.off_by(want[:1], want)
