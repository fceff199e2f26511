"""The example layer: trains, and serves what it computes over whole sequences."""
import os
import runpy

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_layer(capsys):
    runpy.run_path(os.path.join(ROOT, "examples", "state_space_layer.py"), run_name="__main__")
    assert "all good" in capsys.readouterr().out
