"""examples/user_histories.py end to end, in both formats."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("args", [["--users", "40", "--candidates", "7", "--graph-steps", "3"],
                                  ["--users", "3", "--candidates", "1", "--graph-steps", "2", "--fmt", "mx8"]])
def test_user_histories(args):
    spec = importlib.util.spec_from_file_location("user_histories", os.path.join(HERE, "..", "examples", "user_histories.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    worst = example.main(args)
    assert set(worst) == {"whole histories", "step", "candidates", "move"}
    # Weights and outputs are rounded to bf16, each by at most 2^-8 of itself; outputs are means of values that may
    # be a few times larger than the mean.
    assert max(worst.values()) < 2.0 ** -5, worst
