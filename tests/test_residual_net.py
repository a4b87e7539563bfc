"""ResidualNet and its example as far as they go without a GPU."""
import pytest
import torch

import paper_1801_04928_amd as P


def net(**kwargs):
    return P.ResidualNet(2, 40, 24, 4, device="cpu", **kwargs)


def kept(n):
    """What the net keeps for its backward pass."""
    return [*n._sums, *[v._y for v in n.norms], *[v._y for v in n.ups], *[v._z for v in n.ups]]


@pytest.mark.parametrize("dtype, checkpoints", [("f32", "storage"), ("f32", "f32"), ("bf16", "storage"), ("bf16", "bf16"),
                                                ("bf16", torch.bfloat16)])
def test_checkpoints_in_the_storage_type(dtype, checkpoints):
    n = net(dtype=dtype, checkpoints=checkpoints)
    assert all(isinstance(v, torch.Tensor) and v.dtype == n.dtype for v in kept(n))


def test_checkpoints_in_8_bits():
    assert all(isinstance(v, P.E4M3Matrix) for v in kept(net(checkpoints="e4m3")))


@pytest.mark.parametrize("dtype, checkpoints", [("f32", "bf16"), ("bf16", "f32"), ("f32", "e5m2")])
def test_other_checkpoints_are_refused(dtype, checkpoints):
    with pytest.raises(P.LfError):
        net(dtype=dtype, checkpoints=checkpoints)


def test_fewer_bits_only_where_they_are_asked_for():
    """In 8 bits the forward products read what is kept, so the answers change: not by default."""
    assert all(isinstance(v, torch.Tensor) and v.dtype == torch.bfloat16 for v in kept(net()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_steps_add_up(dtype):
    """64 steps of 2^-12 from 1, each a sixteenth of what bf16 tells from 1; every number here is one of bf16's or of fp32's."""
    n = net(dtype=dtype)
    params = [*n.w1, *n.w2, *n.b1, *n.b2, *n.gain]
    for v in params:
        v.fill_(1.0)
    for v in [*n.dw1, *n.dw2, *n.db1, *n.db2, *n.dgain]:
        v.fill_(0.5)
    for _ in range(64):
        n.descend(2.0 ** -11)
    assert all(bool((v == 1 - 2.0 ** -6).all()) for v in params)
    n.w1[0][3, 5] = 2.0                      # a weight of the caller's: it goes on from there, the others where they were
    n.w2[1].copy_(torch.full_like(n.w2[1], 4.0))
    for _ in range(64):
        n.descend(2.0 ** -10)
    assert float(n.w1[0][3, 5]) == 2 - 2.0 ** -5 and bool((n.w2[1] == 4 - 2.0 ** -5).all())
    assert float(n.w1[0][3, 6]) == 1 - 2.0 ** -6 - 2.0 ** -5
