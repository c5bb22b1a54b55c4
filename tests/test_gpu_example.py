"""examples/moe_layer.py: every pass on a stream of its own comes after the work that made its inputs."""
import importlib.util
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_side_streams_wait_for_the_inputs(monkeypatch, capsys):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    spec = importlib.util.spec_from_file_location("moe_layer_example", os.path.join(ROOT, "examples", "moe_layer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    waited, unordered = set(), []
    wait = torch.cuda.Stream.wait_stream

    def wait_stream(self, other):
        waited.add((self.cuda_stream, other.cuda_stream))
        return wait(self, other)

    forward = example.MoELayer.forward

    def checked(self, r, *rest):
        here, home = torch.cuda.current_stream().cuda_stream, torch.cuda.default_stream().cuda_stream
        if here != home and (here, home) not in waited:
            unordered.append(r.shape[0])
        return forward(self, r, *rest)

    monkeypatch.setattr(torch.cuda.Stream, "wait_stream", wait_stream)
    monkeypatch.setattr(example.MoELayer, "forward", checked)
    monkeypatch.setattr(sys, "argv", ["moe_layer.py", "--experts", "8", "--local", "4", "--d", "256", "--f", "256", "--topk", "2"])
    example.main()
    assert "2048 tokens" in capsys.readouterr().out
    assert not unordered
