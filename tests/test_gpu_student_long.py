"""Matrices of more than 2^31 elements: the last rows of a long call are what those rows are elsewhere."""
import pytest
import torch

import paper_1801_04928_amd as P
from tests.student_util import DEV

pytestmark = pytest.mark.gpu


def noise(rows, cols, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    for at in range(0, rows, 8192):
        x[at:at + 8192].normal_(generator=g)
    return x


def test_layer_norm():
    rows, cols, last = 70000, 32768, 5
    x, dy = noise(rows, cols, 1), noise(rows, cols, 2)
    n, short = P.LayerNorm(rows, cols, out="e4m3_128"), P.LayerNorm(last, cols, out="e4m3_128")
    y, want = n.forward(x), short.forward(x[-last:])
    assert torch.equal(y.codes[-last:], want.codes) and torch.equal(y.scales[-last:], want.scales)
    assert torch.equal(n.sum[-last:], short.sum)
    assert torch.equal(n.backward(dy)[-last:], short.backward(dy[-last:]))


def test_blocks():
    rows, cols = 131100, 16500
    x = noise(rows, cols, 3)
    m, t = P.E4M3Blocks(rows, cols, device=DEV), P.E4M3Blocks(cols, rows, device=DEV)
    m.save(x, t)
    at = rows // 128 * 128                                   # the last block's rows
    want, want_t = P.E4M3Blocks(rows - at, cols, device=DEV), P.E4M3Blocks(cols, rows - at, device=DEV)
    want.save(x[at:], want_t)
    groups = -(-cols // 128)
    assert torch.equal(m.codes[at:], want.codes) and torch.equal(m.scales[at:, :groups], want.scales[:, :groups])
    assert torch.equal(t.codes[:, at:], want_t.codes) and torch.equal(t.scales[:, at // 128:at // 128 + 1], want_t.scales[:, :1])
    assert torch.equal(m.load()[at:], want.load())


def test_products():
    """(Rows at either end, of one kernel: a short call might split its contraction.)"""
    rows, outputs, inputs, last = 140000, 16400, 200, 300
    x, w, dy = noise(rows, inputs, 4), noise(outputs, inputs, 5), noise(rows, outputs, 6)
    x[-last:], dy[-last:] = x[:last], dy[:last]
    n = P.BlockLinear(rows, outputs, inputs, act="relu", z="bf16")
    n.set_params(w)
    y = n.forward(x)
    assert torch.equal(y[-last:], y[:last]) and torch.equal(n.z[-last:], n.z[:last]) and bool((n.z[:last] != 0).any())
    dx = n.backward(dy)
    assert torch.equal(dx[-last:], dx[:last]) and bool((dx[:last] != 0).any())


def test_distillation():
    rows, classes, top, last = 33000, 65601, 9, 7
    z, t = noise(rows, classes, 7), noise(rows, top, 8)
    k = torch.randint(0, classes, (rows, top), dtype=torch.int32, device=DEV)
    n, short = P.Distillation(rows, classes, top, temperature=2.0), P.Distillation(last, classes, top, temperature=2.0)
    loss, want = n.forward(z, t, k), short.forward(z[-last:], t[-last:], k[-last:])
    assert torch.equal(loss[-last:], want) and torch.equal(n.dlogits[-last:], short.dlogits)


def test_layer_norm_backward_of_more_rows_than_a_launch_takes():
    """A workgroup a row, 2^20 of them a launch: the rows at the borders of the launches, of a sum in either form."""
    torch.cuda.empty_cache()
    part, cols = 1 << 20, 8193
    rows = 4 * part + 3
    x = noise(rows, cols, 9)                                 # (both the gradient and the sum)
    mean, rstd = torch.randn(rows, device=DEV), torch.rand(rows, device=DEV)
    m = P.E4M3Matrix(rows, cols, device=DEV).save(x)
    at = torch.tensor([0, 1, *(i * part + j for i in (1, 2, 3, 4) for j in (-2, -1, 0, 1)), rows - 1], device=DEV)
    n, short = P.LayerNorm(rows, cols, passes="backward"), P.LayerNorm(len(at), cols, passes="backward")
    for stored, few in ((x, x[at]), (m, P.E4M3Matrix.of(m.codes[at], m.scales[at], cols))):
        n._dx.fill_(77)
        dx = n.backward(x, stored=stored, mean=mean, rstd=rstd)
        assert torch.equal(dx[at], short.backward(x[at], stored=few, mean=mean[at], rstd=rstd[at]))
        assert all(not bool((v == 77).all(1).any()) for v in dx.split(part))
    del x, m, n, dx, stored
    torch.cuda.empty_cache()
