"""ResidualNet and its example on the GPU."""
import importlib.util
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_residual_net", os.path.join(ROOT, "examples", "train_residual_net.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("checkpoints", ["e4m3", "storage"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_example_takes_its_options(dtype, checkpoints, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["train_residual_net.py", "--depth", "1", "--width", "64", "--hidden", "64", "--rows", "32",
                                      "--steps", "3", "--dtype", dtype, "--checkpoints", checkpoints])
    example().main()
    out = capsys.readouterr().out
    assert "step 2: cost" in out and "one sample" in out
