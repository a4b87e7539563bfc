"""The activations of the product's epilogue and their slopes on the GPU, relative to their own size: what saturates and what is
far out in a tail keeps its digits.

u = 2^-24 is half a step of fp32.  exponential(x) multiplies x by log2(e) (the constant is off by 0.22 u of itself, the product
is rounded: together 1.25 |x| u of the result) and takes an instruction good to an ulp (2 u): (1.25 |x| + 3) u.  gelu's argument z^2 / 2
is rounded before that: (2.25 z^2 / 2 + 3) u.  Reciprocals are good to an ulp, sums and products to u; the tail's fit is off by
0.54 u, 3 u as evaluated.  Numbers below 2^-126 may be lost where they come up: 2^-125, times what they are multiplied by."""
import math

import numpy as np
import pytest
import torch

import paper_1801_04928_amd as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"


def sigma(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1 / (1 + e), e / (1 + e))


def phi(z):
    return np.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def normal(z):
    return 0.5 * np.vectorize(math.erfc)(-z / math.sqrt(2))


def value(name, z):
    """(the activation, how far off it may be)"""
    below = np.maximum(-z, 0)
    floor = 2.0 ** -125 * np.maximum(np.abs(z), 1)
    if name == "relu":
        return np.maximum(z, 0), np.zeros_like(z)
    if name == "gelu":
        y = z * normal(z)
        return y, (1.125 * below ** 2 + 18) * U * np.abs(y) + floor
    y = sigma(z) * (z if name == "silu" else 1)
    return y, (1.25 * below + 10) * U * np.abs(y) + floor


def slope(name, z):
    """(its slope, how far off it may be: relative to the sum of its terms' sizes)"""
    floor = 2.0 ** -125 * np.maximum(np.abs(z), 1)
    if name == "relu":
        return (z > 0) * 1.0, np.zeros_like(z)
    if name == "gelu":
        a, b = np.abs(z) * phi(z), normal(z)
        return z * phi(z) + b, U * ((1.125 * z * z + 24) * a + (1.125 * np.maximum(-z, 0) ** 2 + 24) * b) + floor
    s, rest = sigma(z), sigma(-z)
    if name == "sigmoid":
        return s * rest, (1.25 * np.abs(z) + 12) * U * s * rest + floor
    return s * (1 + z * rest), (1.25 * np.maximum(-z, 0) + 24) * U * s * (1 + np.abs(z) * rest) + floor


POINTS = np.concatenate([np.linspace(-14, 14, 2801), np.linspace(-100, 100, 1601), [1e-30, -1e-30, 1e-6, -1e-6, 300.0, -300.0]])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["sigmoid", "relu", "silu", "gelu"])
def test_activations_and_slopes_keep_their_digits(name, dtype):
    """One input and a weight of one: y is the activation of x and dx its slope, each rounded once (dz, too, in bf16: dx holds it)."""
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    x = torch.from_numpy(POINTS).to(t).to(DEV)[:, None].contiguous()
    z, n = x[:, 0].double().cpu().numpy(), len(POINTS)
    p = P.Linear(n, 1, 1, dtype, act=name, z=dtype, device=DEV)
    p.set_params(torch.ones(1, 1, dtype=t, device=DEV))
    y = p.forward(x).double().cpu().numpy()[:, 0]
    dx = p.backward(torch.ones_like(x), x).double().cpu().numpy()[:, 0]
    half = 0.0 if dtype == "f32" else 2.0 ** -8
    for what, got, (want, off) in (("value", y, value(name, z)), ("slope", dx, slope(name, z))):
        # (bf16 numbers below 2^-126 may be lost in the product)
        bound = off + half * (np.abs(want) + off) + (2.0 ** -126 if half else 0)
        worst = int(np.argmax(np.abs(got - want) - bound))
        assert (np.abs(got - want) <= bound).all(), f"{what} of {name} at {z[worst]}: {got[worst]} for {want[worst]}, {bound[worst]:.3g} allowed"
