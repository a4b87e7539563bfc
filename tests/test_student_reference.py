"""The references of the student nets' operators against differences and definitions written another way."""
import math

import pytest
import torch

from tests import student_reference as R


def rand(*shape, seed=0):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def differences(f, x, step=1e-6):
    g = torch.zeros_like(x)
    for i in range(x.numel()):
        e = torch.zeros_like(x).view(-1)
        e[i] = step
        e = e.view(x.shape)
        g.view(-1)[i] = (f(x + e) - f(x - e)) / (2 * step)
    return g


def test_norm_gradients():
    """Against central differences of step h = 1e-6: off by h^2 of third derivatives and 1e-16 / h of the sum's values."""
    x, gain, shift, dy, dsum = rand(3, 7), rand(7, seed=1), rand(7, seed=2), rand(3, 7, seed=3), rand(3, 7, seed=4)

    def total(x, gain, shift):
        r = R.norm_forward(x, None, gain, shift, 1e-3)
        return float((r["y"][0] * dy).sum() + (x * dsum).sum())

    f = R.norm_forward(x, None, gain, shift, 1e-3)
    b = R.norm_backward(dy, x, gain, f["mean"][0], f["rstd"][0], dsum)
    for got, want in ((b["dx"][0], differences(lambda v: total(v, gain, shift), x)),
                      (b["dgain"][0], differences(lambda v: total(x, v, shift), gain)),
                      (b["dshift"][0], differences(lambda v: total(x, gain, v), shift))):
        assert float((got - want).abs().max()) < 1e-7


def test_distillation_gradient():
    z, t = rand(3, 9), rand(3, 4, seed=1)
    classes = torch.tensor([[0, 3, 8, 5], [2, 2, -1, 7], [1, 0, 4, 6]])
    weight = torch.tensor([0.5, 2.0, 0.0], dtype=torch.float64)
    for T in (0.5, 1.0, 3.0):
        got = R.distil(z, t, classes, T, weight)["dlogits"][0]
        want = differences(lambda v: float(R.distil(v, t, classes, T, weight)["loss"][0].sum()), z)
        assert float((got - want).abs().max()) < 1e-7 and bool((got[2] == 0).all())


def test_distillation_of_equal_distributions_is_nothing():
    z = rand(2, 6)
    classes = torch.arange(6).repeat(2, 1)
    r = R.distil(z, z.clone(), classes, 2.0, torch.ones(2, dtype=torch.float64))
    assert float(r["loss"][0].abs().max()) < 1e-14 and float(r["dlogits"][0].abs().max()) < 1e-14


def test_codes_are_torchs():
    """... which rounds to nearest, ties to even, too."""
    v = torch.cat([rand(4000) * 100, torch.linspace(-448, 448, 7169, dtype=torch.float64), torch.linspace(-0.07, 0.07, 4097, dtype=torch.float64)])
    v = v.float().double()
    assert torch.equal(R.nearest_codes(v), v.float().to(torch.float8_e4m3fn).double())


def test_scales_are_the_least_that_hold_a_group():
    v = rand(5, 300) * torch.exp2(torch.arange(5, dtype=torch.float64) * 20 - 40)[:, None]
    v[1, 128:256] = 0
    v[2, 7], v[2, 130] = math.inf, math.nan
    codes, e = R.pack(v)
    assert bool((codes.nan_to_num().abs() <= 448).all()) and bool(codes[2, 7].isnan()) and bool(codes[2, 130].isnan())
    assert int(e[1, 1]) == -117
    for r in range(5):
        for g in range(3):
            part = v[r, 128 * g:128 * g + 128]
            top = float(part[part.isfinite()].abs().max())
            assert top <= 448 * 2.0 ** int(e[r, g]) and (int(e[r, g]) == -117 or top > 448 * 2.0 ** (int(e[r, g]) - 1))
    codes, e = R.pack_tiles(v[:, :200])
    assert e.shape == (1, 2) and torch.equal(R.held_tiles(v[:, :200])[3], R.unpack(codes, e)[3])


@pytest.mark.parametrize("name", ["none", "sigmoid", "relu", "silu", "gelu"])
def test_slopes(name):
    z = rand(40) * 3
    want = (R.act(z + 1e-6, name) - R.act(z - 1e-6, name)) / 2e-6
    assert float((R.slope(z, name) - want).abs().max()) < 1e-8


def test_the_bound_of_sums_in_14_bits_holds_its_worst_case():
    """One large product and seven small ones just below what is kept."""
    x, w = torch.full((1, 8), 2.0 ** -7, dtype=torch.float64), torch.full((1, 8), 2.0 ** -7, dtype=torch.float64)
    x[0, 0] = w[0, 0] = 1.0
    z, bound = R.product(x, w, exact=False)
    assert float(z) - 1 <= float(bound)
