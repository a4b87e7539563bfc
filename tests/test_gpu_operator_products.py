"""Every kernel of the products on the GPU, against the products in 64 bits, at sizes with ends in every direction (test_operators_routes
holds that these are the kernels that run).

All matrices lie inside larger ones, at odd addresses: what surrounds an input is NaN, and so are the codes past a row's end; what
surrounds an output must stay.  Tolerances as in test_gpu_operators: a sum of n products in fp32 is off by at most n u of the
sum of their magnitudes, u = 2^-24; the last rounding is half a step of its type; 8 bits are off by 2^-4 of the value or 2^-10 of the
scale.  relu's slope is 0 or 1: dz is exact."""
import pytest
import torch

import paper_1801_04928_amd as P
from paper_1801_04928_amd import operators as ops
from tests import operator_routes as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
MARK = 77.0
DEV = "cuda:0"


class Framed:
    """A matrix inside a larger one of NaN (an input: its values are given) or of a mark (an output)."""

    def __init__(self, rows, cols, t, values=None):
        self.shape = (rows, cols)
        self.all = torch.full((rows + 2, cols + 3), MARK if values is None else float("nan"), dtype=t, device=DEV)
        self.t = self.all[1:rows + 1, 1:cols + 1]
        if values is not None:
            self.t.copy_(values)
        self.m = ops._matrix("m", self.t, self.shape, 0, P.lf_matrix())

    def values(self):
        return self.t.double()

    def check(self, name, want, off):
        got = self.values()
        bound = off + HALF[self.t.dtype] * (want.abs() + off) + 1e-30
        far = (got - want).abs() - bound
        assert bool((far <= 0).all()), f"{name}: {int((~(far <= 0)).sum())} values off, the first at {(~(far <= 0)).nonzero()[0].tolist()}"
        self.t.fill_(MARK)
        assert bool((self.all == MARK).all()), f"{name}: written outside"


class FramedEight:
    """The same in 8 bits."""

    def __init__(self, rows, cols, values=None):
        self.shape, groups = (rows, cols), -(-cols // 32)
        self.codes = torch.full((rows + 1, groups * 32 + 32), 0x7f, dtype=torch.uint8, device=DEV)
        self.scales = torch.full((rows + 1, groups + 3), 255, dtype=torch.uint8, device=DEV)
        self.e = P.E4M3Matrix.of(self.codes[:rows, :groups * 32], self.scales[:rows, :groups], cols)
        if values is not None:
            self.e.save(values)
            self.codes[:, cols:] = 0x7f
        self.m = self.e._m

    def values(self):
        return self.e.load(dtype="f32").double()

    def check(self, name, want, off):
        rows, cols = self.shape
        scale = torch.exp2(self.e.scales.double() - 127).repeat_interleave(32, 1)[:, :cols]
        bound = off + torch.maximum(2.0 ** -4 * (want.abs() + off), 2.0 ** -10 * scale)
        assert bool(((self.values() - want).abs() <= bound).all()), name
        assert bool((self.e.codes[:, cols:] == 0).all()), f"{name}: codes past the last column are zero"
        self.e.codes.fill_(0x7f)
        self.e.scales.fill_(255)
        assert bool((self.codes == 0x7f).all()) and bool((self.scales == 255).all()), f"{name}: written outside"


def matrix(rows, cols, t, eight, values=None):
    return FramedEight(rows, cols, values) if eight else Framed(rows, cols, t, values)


def product(p, q):
    """p q^T in 64 bits, of operands laid out whole."""
    return torch.mm(p.contiguous(), q.t().contiguous())


def scratch(nbytes):
    return torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)


def sum_off(n, p, q):
    return (n + 8) * U * product(p.abs(), q.abs())


@pytest.mark.parametrize("case", [c for c, _ in R.CASES], ids=lambda c: "-".join(map(str, c)))
def test_products(case):
    what, rows, o, i, dtype, kept = case
    t, dt = TYPE[dtype], P.LF_F32 if dtype == "f32" else P.LF_BF16
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + 3 * o + 7 * i)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device=DEV) * std).to(t)

    x, w = matrix(rows, i, t, "x" in kept, normal(rows, i)), Framed(o, i, t, normal(o, i, std=i ** -0.5))
    b = torch.randn(o, generator=g, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    xv, wv = x.values(), w.values()
    if what == "forward":
        residual, y, z = Framed(rows, o, t, normal(rows, o)), Framed(rows, o, t), matrix(rows, o, t, "z" in kept)
        nbytes = P.lf_linear_workspace_bytes(rows, o, i, dt)
        s = scratch(nbytes)
        status = P.lf_linear_forward(rows, o, i, x.m, w.m, b.data_ptr(), P.LF_ACT_RELU, residual.m, y.m, z.m, s.data_ptr(), nbytes, stream)
        assert status == P.LF_OK, P.lf_operator_error()
        want = product(xv, wv) + b.double()
        off = sum_off(i, xv, wv) + (i + 8) * U * b.double().abs()
        r = residual.values()
        y.check("y", want.clamp(min=0) + r, off + U * (want.abs() + r.abs()))
        z.check("z", want, off)
    else:
        z, dy = matrix(rows, o, t, "z" in kept, normal(rows, o)), Framed(rows, o, t, normal(rows, o))
        dx, dw = Framed(rows, i, t) if what != "dw" else None, Framed(o, i, torch.float32) if what != "dx" else None
        db = torch.full((o + 2,), MARK, device=DEV)
        nbytes = P.lf_linear_backward_workspace_bytes(rows, o, i, dt)
        s = scratch(nbytes)
        status = P.lf_linear_backward(rows, o, i, dy.m, z.m, P.LF_ACT_RELU, x.m if dw else None, w.m if dx else None, dx.m if dx else None,
                                      dw.m if dw else None, db[1:].data_ptr() if what == "backward" else 0, s.data_ptr(), nbytes, stream)
        assert status == P.LF_OK, P.lf_operator_error()
        dz = torch.where(z.values() > 0, dy.values(), 0.0)
        if dx:
            dx.check("dx", product(dz, wv.t()), sum_off(o, dz, wv.t()))
        if dw:
            dw.check("dw", product(dz.t(), xv.t()), sum_off(rows, dz.t(), xv.t()))
        if what == "backward":
            off = (rows + 12) * U * dz.abs().sum(0) + 1e-30
            assert bool(((db[1:-1].double() - dz.sum(0)).abs() <= off).all()), "db"
            db[1:-1] = MARK
        assert bool((db == MARK).all()), "db: written outside"
    assert bool((s[nbytes:] == 255).all()), "written past the workspace"
