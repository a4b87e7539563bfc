"""ResidualNet with layer norms, products in blocks of 128 and classes, as far as it goes without a GPU."""
import pytest
import torch

import paper_1801_04928_amd as P


def net(**kwargs):
    return P.ResidualNet(2, 40, 24, 4, device="cpu", **kwargs)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("checkpoints", ["storage", "e4m3"])
def test_what_is_kept(dtype, checkpoints):
    n = net(dtype=dtype, checkpoints=checkpoints, norm="layer", products="e4m3_128", classes=30)
    kind = P.E4M3Matrix if checkpoints == "e4m3" else torch.Tensor
    assert all(isinstance(v, kind) for v in n._sums) and len(n._sums) == 3
    assert all(isinstance(p._z, P.E4M3Blocks if checkpoints == "e4m3" else torch.Tensor) for p in n.ups)
    assert all(isinstance(p._x_t, P.E4M3Blocks) and p._x_t.shape == (p.inputs, 4) for p in (*n.ups, *n.downs, n.head))
    assert all(m._y is n.norms[0]._y for m in n.norms) and n.out.shape == (4, 30)
    assert len(n.gain) == len(n.shift) == len(n.dshift) == 3 and all(isinstance(m, P.LayerNorm) for m in n.norms)


def test_a_net_for_answers_keeps_nothing():
    n = net(norm="layer", products="e4m3_128", classes=30, passes="forward")
    assert all(isinstance(v, P.E4M3Blocks) for v in (*(m._y for m in n.norms), *(p._y for p in n.ups)))
    assert all(s is n._s for s in n._sums) and all(p._z is None and p._x_t is None and p.dw is None for p in (*n.ups, *n.downs, n.head))
    with pytest.raises(P.LfError, match="distil"):
        n.distil(torch.zeros(4, 40), torch.zeros(4, 3), torch.zeros(4, 3, dtype=torch.int32))
    with pytest.raises(P.LfError, match="distil"):
        net().distil(torch.zeros(4, 40), torch.zeros(4, 3), torch.zeros(4, 3, dtype=torch.int32))


@pytest.mark.parametrize("change", [dict(norm="batch"), dict(products="e4m3"), dict(passes="backward"), dict(classes=0), dict(classes=-3)])
def test_refusals(change):
    with pytest.raises(P.LfError):
        net(**change)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_parameter_descends(dtype):
    """... in steps that bf16 alone would not tell from nothing; every number here is one of bf16's or of fp32's."""
    n = net(dtype=dtype, norm="layer", products="e4m3_128", classes=30)
    params = [*n.w1, *n.w2, n.w_out, *n.b1, *n.b2, n.b_out, *n.gain, *n.shift]
    grads = [*n.dw1, *n.dw2, n.dw_out, *n.db1, *n.db2, n.db_out, *n.dgain, *n.dshift]
    for v in params:
        v.fill_(1.0)
    for v in grads:
        v.fill_(0.5)
    n._stale = False
    for _ in range(64):
        n.descend(2.0 ** -11)
    assert all(bool((v == 1 - 2.0 ** -6).all()) for v in params) and n._stale


def test_teachers_of_no_matrix_are_refused():
    for t in (torch.zeros(()), torch.zeros(4), torch.zeros(4, 3, 1)):
        with pytest.raises(P.LfError, match="top_logits"):
            net(classes=30).distil(torch.zeros(4, 40), t, torch.zeros(4, 3, dtype=torch.int32))


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("kinds", [dict(), dict(checkpoints="e4m3"), dict(products="e4m3_128")])
def test_a_net_for_answers_has_one_block_s_activations(kinds, norm):
    n = P.ResidualNet(5, 40, 24, 4, device="cpu", norm=norm, passes="forward", classes=30, **kinds)
    assert len({id(m._y) for m in n.norms}) == len({id(p._y) for p in n.ups}) == len({id(p._y) for p in n.downs}) == 1
    assert all(p._z is None for p in n.ups)


def test_a_net_for_answers_does_not_learn():
    n = net(passes="forward")
    with pytest.raises(P.LfError, match="descend"):
        n.descend(0.5)
    with pytest.raises(P.LfError, match="backward"):
        n.backward(torch.zeros(4, 40, dtype=torch.bfloat16))
