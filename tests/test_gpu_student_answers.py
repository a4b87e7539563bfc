"""Nets for answers, whose blocks write to the same memory, answer as those that keep every block's activations."""
import pytest
import torch

import paper_1801_04928_amd as P
from tests.student_util import DEV, TYPE, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoints", ["storage", "e4m3"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_answers_of_four_blocks(norm, checkpoints, dtype):
    nets = [P.ResidualNet(4, 72, 136, 150, dtype=dtype, norm=norm, checkpoints=checkpoints, classes=45, passes=passes) for passes in ("both", "forward")]
    x = values(1, 150, 72).to(TYPE[dtype]).to(DEV)
    for net in nets:
        net.init(2)
    for n in (150, 1, 131):
        assert torch.equal(nets[0].forward(x[:n]), nets[1].forward(x[:n]))
