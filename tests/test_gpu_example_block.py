"""examples/decoder_block.py runs, prompts and decode steps, with small sizes."""
import importlib.util
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_it_runs(monkeypatch, capsys):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    spec = importlib.util.spec_from_file_location("decoder_block_example", os.path.join(ROOT, "examples", "decoder_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    monkeypatch.setattr(sys, "argv", ["decoder_block.py", "--heads", "4", "--kv-heads", "2", "--d", "256", "--f", "256", "--experts", "4",
                                      "--prompt", "77", "--sequences", "3", "--steps", "5"])
    example.main()
    assert "5 steps of 3 sequences" in capsys.readouterr().out
