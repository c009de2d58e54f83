"""The serving example: append, attention, fork, free, compact, copy and the migration of a 4-bit cache in one program."""
import os
import runpy

import pytest

pytestmark = pytest.mark.gpu


def test_serve_and_switch(capsys):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_and_switch.py")
    runpy.run_path(path, run_name="__main__")
    assert "same outputs" in capsys.readouterr().out
