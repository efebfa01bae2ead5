"""The example of the block's operators runs: one pass of one token and of a batch, and a training loss that falls."""
import os
import runpy
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_serves_and_learns(monkeypatch):
    monkeypatch.setattr(sys, "argv", ["int8_ffn_block.py", "--tokens", "300", "--width", "192", "--hidden", "512",
                                      "--steps", "10"])
    losses = runpy.run_path(os.path.join(ROOT, "examples", "int8_ffn_block.py"))["main"]()
    assert len(losses) == 10 and losses[-1] < 0.95 * losses[0]
