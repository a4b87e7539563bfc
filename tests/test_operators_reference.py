"""The 64-bit reference of the residual blocks' operators, held against other statements of the same: torch's e4m3 type for
the codes, differences of the forward pass for every gradient."""
import numpy as np
import pytest
import torch

from tests import operators_reference as R


def test_codes_are_torchs_e4m3():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(want), np.isnan(R.TABLE)) and np.array_equal(want[~np.isnan(want)], R.TABLE[~np.isnan(R.TABLE)])
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 20000), rng.uniform(-0.1, 0.1, 20000), (R.TABLE[:126] + R.TABLE[1:127]) / 2,
                        [0.0, -0.0, 448.0, -448.0, 2.0 ** -10, 2.0 ** -9]]).astype(np.float32)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.nearest_code(v.astype(np.float64)), want)


def test_scale_is_the_least_that_holds_the_group():
    x = np.zeros((6, 32))
    x[0, 3], x[1, 0], x[2, 5], x[3, 31], x[4, 1] = 448.0, 448.001, -1.0, 2.0 ** -130, np.inf
    codes, scales = R.to_eight(x)
    assert [int(s) - 127 for s in scales[:, 0]] == [0, 1, -8, -117, -117, -117]
    assert codes[4, 1] == 0x7f and codes[2, 5] == 0x80 | 0x78
    back = R.from_eight(codes, scales)
    assert back[0, 3] == 448 and back[2, 5] == -1


def differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + h
        up = f()
        x[i] = old - h
        down = f()
        x[i] = old
        g[i] = (up - down) / (2 * h)
    return g


@pytest.mark.parametrize("with_dsum", [False, True])
def test_norm_gradients_are_differences(with_dsum):
    rng = np.random.default_rng(1)
    x, branch, gain = rng.normal(size=(3, 5)), rng.normal(size=(3, 5)), rng.normal(size=5)
    wy, ws = rng.normal(size=(3, 5)), rng.normal(size=(3, 5)) * with_dsum

    def cost():
        s, _, y = R.norm_forward(x, branch, gain, 1e-3)
        return (wy * y).sum() + (ws * s).sum()
    s, rstd, _ = R.norm_forward(x, branch, gain, 1e-3)
    dx, dgain = R.norm_backward(wy, s, gain, rstd, ws if with_dsum else None)
    for got, of in ((dx, x), (dx, branch), (dgain, gain)):
        assert np.abs(got - differences(cost, of)).max() < 1e-7


@pytest.mark.parametrize("name", ["none", "sigmoid", "relu", "silu", "gelu"])
def test_product_gradients_are_differences(name):
    rng = np.random.default_rng(2)
    x, w, b, r = rng.normal(size=(4, 3)), rng.normal(size=(5, 3)), rng.normal(size=5), rng.normal(size=(4, 5))
    wy = rng.normal(size=(4, 5))

    def cost():
        return (wy * R.linear_forward(x, w, b, name, r)[1]).sum()
    z, _ = R.linear_forward(x, w, b, name, r)
    assert name != "relu" or np.abs(z).min() > 1e-3           # no kink within a difference
    dz, dx, dw, db = R.linear_backward(wy, z, name, x, w)
    for got, of in ((dx, x), (dw, w), (db, b), (wy, r)):
        assert np.abs(got - differences(cost, of)).max() < 1e-7
