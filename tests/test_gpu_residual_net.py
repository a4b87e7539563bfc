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


@pytest.mark.parametrize("checkpoints", ["e4m3", "storage"])
def test_a_pass_of_no_rows(checkpoints):
    """Nothing comes out, and the gradients, sums over no rows, are zeros whatever was there."""
    import torch
    import paper_1801_04928_amd as P
    net = P.ResidualNet(2, 40, 24, 4, checkpoints=checkpoints)
    net.init()
    grads = [*net.dw1, *net.dw2, *net.db1, *net.db2, *net.dgain]
    for g in grads:
        g.fill_(7.0)
    x = torch.ones(4, 40, dtype=torch.bfloat16, device="cuda:0")[:0]
    assert net.forward(x).shape == (0, 40) and net.backward(x).shape == (0, 40)
    assert all(bool((g == 0).all()) for g in grads)
