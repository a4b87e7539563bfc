"""Where a matrix lies does not change a result: bits of every output, whatever element of 16 bytes its rows and its inputs' rows begin at."""
import pytest
import torch

import paper_1801_04928_amd as P
from paper_1801_04928_amd import operators as ops

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


class At:
    """Matrices `off` elements into their memory, with rows `off` elements apart from one another; NaN around them."""

    def __init__(self, off):
        self.off = off

    def __call__(self, values):
        rows, cols = values.shape
        around = torch.full((rows + 1, cols + 2 * self.off), float("nan"), dtype=values.dtype, device=DEV)
        t = around[:rows, self.off:self.off + cols]
        t.copy_(values)
        return t

    def matrix(self, values):
        t = self(values)
        return t, ops._matrix("m", t, tuple(t.shape), 0, P.lf_matrix())


def normal(t, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(shape))
    return torch.randn(*shape, generator=g, device=DEV).to(t)


def call(status):
    assert status == P.LF_OK, P.lf_operator_error()


def linear(at, rows, o, i, t, kept):
    x, w, residual, dy = (normal(t, *s) for s in ((rows, i), (o, i), (rows, o), (rows, o)))
    dt = P.LF_F32 if t == torch.float32 else P.LF_BF16
    e = P.E4M3Matrix(rows, i, device=DEV).save(x) if kept else None
    xt, mx = (e, e._m) if kept else at.matrix(x)
    (y, my), (z, mz), (dx, mdx), (dw, mdw) = (at.matrix(torch.zeros_like(v)) for v in (residual, residual, x, w))
    (wt, mw), (rt, mr), (dyt, mdy) = (at.matrix(v) for v in (w, residual, dy))
    b, db = normal(torch.float32, o), torch.zeros(o, device=DEV)
    nbytes = max(P.lf_linear_workspace_bytes(rows, o, i, dt), P.lf_linear_backward_workspace_bytes(rows, o, i, dt), 256)
    s = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)
    call(P.lf_linear_forward(rows, o, i, mx, mw, b.data_ptr(), P.LF_ACT_SILU, mr, my, mz, s.data_ptr(), nbytes))
    call(P.lf_linear_backward(rows, o, i, mdy, mz, P.LF_ACT_SILU, mx, mw, mdx, mdw, db.data_ptr(), s.data_ptr(), nbytes))
    torch.cuda.synchronize()
    return [v.clone() for v in (y, z, dx, dw, db)]


def norm(at, rows, cols, t, kept):
    x, branch, dy, dsum = (normal(t, rows, cols) + k for k in range(4))
    (xt, mx), (bt, mb), (dyt, mdy), (dst, mds) = (at.matrix(v) for v in (x, branch, dy, dsum))
    (total, ms), (y, my), (dx, mdx) = (at.matrix(torch.zeros_like(x)) for _ in range(3))
    e = P.E4M3Matrix(rows, cols, device=DEV)
    gain, rstd, dgain = 1 + normal(torch.float32, cols) / 8, torch.zeros(rows, device=DEV), torch.zeros(cols, device=DEV)
    nbytes = max(P.lf_norm_workspace_bytes(rows, cols), 256)
    s = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)
    call(P.lf_norm_forward(rows, cols, mx, mb, gain.data_ptr(), 1e-6, ms, my, rstd.data_ptr()))
    e.save(total)
    loaded = at(torch.zeros_like(x))
    e.load(out=loaded)
    call(P.lf_norm_backward(rows, cols, mdy, e._m if kept else ms, gain.data_ptr(), rstd.data_ptr(), mds, mdx, dgain.data_ptr(),
                            s.data_ptr(), nbytes))
    torch.cuda.synchronize()
    return [v.clone() for v in (total, y, rstd, e.codes, e.scales, loaded, dx, dgain)]


@pytest.mark.parametrize("kept", [False, True], ids=["stored", "8bit"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 40, 64), (1, 333, 1030), (2, 45, 520), (3, 45, 2500), (5, 70, 130), (70, 130, 300), (130, 72, 4100)], ids=str)
def test_products(shape, dtype, kept):
    want = linear(At(0), *shape, TYPE[dtype], kept)
    for off in range(1, 8):
        for name, a, b in zip(("y", "z", "dx", "dw", "db"), linear(At(off), *shape, TYPE[dtype], kept), want):
            assert torch.equal(a, b), (name, off)


@pytest.mark.parametrize("kept", [False, True], ids=["stored", "8bit"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 7), (1, 40), (1, 1500), (9, 64), (3, 5000), (2, 12000), (2, 20000), (300, 100)], ids=str)
def test_norms_and_8_bits(shape, dtype, kept):
    want = norm(At(0), *shape, TYPE[dtype], kept)
    for off in range(1, 8):
        for name, a, b in zip(("sum", "y", "rstd", "codes", "scales", "loaded", "dx", "dgain"), norm(At(off), *shape, TYPE[dtype], kept), want):
            assert torch.equal(a, b), (name, off)
