"""The example runs, and its accepted nodes agree with decode steps."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("argv", [["--prompt", "1000"], ["--prompt", "333", "--samples", "1", "--nodes", "5", "--rounds", "4"],
                                  ["--prompt", "2000", "--samples", "3", "--nodes", "70", "--rounds", "5"]])
def test_tree_decoding(argv):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tree_decoding.py")
    spec = importlib.util.spec_from_file_location("tree_decoding", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main(argv) > 0
