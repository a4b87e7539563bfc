"""Matrices in 8 bits with scales that this library does not write: every byte stands for 2^(byte - 127), 255 for a NaN."""
import numpy as np
import pytest
import torch

import paper_1801_04928_amd as P
from tests import operators_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def every(first, last, numbers=False):
    """(matrix, its values in 64 bits): row r has scale byte first + r and all 256 codes; numbers: zeros for the two that are none."""
    codes, bytes_ = np.tile(np.arange(256, dtype=np.uint8), (last - first, 1)), np.arange(first, last)
    if numbers:
        codes[:, 0x7f] = codes[:, 0xff] = 0
    values = R.TABLE[codes] * 2.0 ** (bytes_[:, None] - 127.0)
    values[bytes_ == 255] = np.nan
    scales = torch.from_numpy(bytes_.astype(np.uint8))[:, None].repeat(1, 8)
    return P.E4M3Matrix.of(torch.from_numpy(codes).to(DEV), scales.to(DEV), 256), torch.from_numpy(values)


def same(got, values):
    """Each value rounded once (from 64 bits to 32 nothing is lost but what is above the largest number)."""
    want = values.float().to(got.dtype)
    got = got.cpu()
    return bool(((got == want) | (got.isnan() & want.isnan())).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loaded(dtype):
    m, values = every(0, 256)
    assert same(m.load(dtype=dtype), values)


# (few rows, and tiles; scales whose largest values are finite, so that nothing times zero is a NaN)
@pytest.mark.parametrize("first, last", [(0, 3), (7, 11), (0, 247), (245, 247)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_operand_of_a_product(first, last, dtype):
    m, values = every(first, last, numbers=True)
    p = P.Linear(last - first, 256, 256, dtype, device=DEV)
    p.set_params(torch.eye(256, device=DEV).to(TYPE[dtype]))
    assert same(p.forward(m), values)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_scale_that_is_none_spoils_its_row(rows, dtype):
    m, _ = every(200 - rows, 200, numbers=True)
    m.scales[rows // 2, 3] = 255
    p = P.Linear(rows, 256, 256, dtype, device=DEV)
    p.set_params(torch.eye(256, device=DEV).to(TYPE[dtype]))
    spoiled = p.forward(m).isnan()
    assert bool(spoiled[rows // 2].all()) and int(spoiled.sum()) == 256


@pytest.mark.parametrize("byte", [0, 1, 9, 10, 127, 200, 255])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_stored_sum_of_a_norm(byte, dtype):
    """One row with rstd = 1 and dy = 1: the gain's gradient is the sum itself."""
    m, values = every(byte, byte + 1, numbers=True)
    n = P.RmsNorm(1, 256, dtype, passes="backward", device=DEV)
    n.backward(torch.ones(1, 256, device=DEV, dtype=TYPE[dtype]), stored=m, rstd=torch.ones(1, device=DEV))
    assert same(n.dgain, values[0])
