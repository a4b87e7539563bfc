"""A NaN next to an operand's ends reaches the sums that it is part of and no others, in every kernel of the products.  (What a tile has past
an end is loaded from inside the matrix, the last rows and columns among it, and must leave nothing behind.)"""
import pytest
import torch

import paper_1801_04928_amd as P
from tests import operator_routes as R
from tests.test_gpu_operator_products import DEV, MARK, TYPE, Framed, FramedEight, matrix

pytestmark = pytest.mark.gpu


def spoil(m, row, col):
    if isinstance(m, FramedEight):
        m.codes[row, col] = 0xff
    else:
        m.t[row, col] = float("nan")


def only(name, m, rows=(), cols=()):
    """NaN are these rows and columns."""
    got = m.values().isnan()
    want = torch.zeros_like(got)
    for r in rows:
        want[r] = True
    for c in cols:
        want[:, c] = True
    assert torch.equal(got, want), f"{name}: {int((got & ~want).sum())} too many, {int((want & ~got).sum())} too few"


@pytest.mark.parametrize("case", [c for c, _ in R.CASES], ids=lambda c: "-".join(map(str, c)))
def test_spoiled_ends(case):
    what, rows, o, i, dtype, kept = case
    t, dt = TYPE[dtype], P.LF_F32 if dtype == "f32" else P.LF_BF16
    g = torch.Generator(device=DEV)
    g.manual_seed(1)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV).to(t)

    x, w = matrix(rows, i, t, "x" in kept, normal(rows, i)), Framed(o, i, t, normal(o, i))
    r0, r1, c0, c1, n0, n1 = 0, rows - 1, 0, i - 1, 0, o - 1
    if what == "forward":
        spoil(x, r1, c1)
        w.t[n1, c0] = float("nan")
        y, z = Framed(rows, o, t), matrix(rows, o, t, "z" in kept)
        nbytes = P.lf_linear_workspace_bytes(rows, o, i, dt)
        s = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
        assert P.lf_linear_forward(rows, o, i, x.m, w.m, 0, P.LF_ACT_SIGMOID, None, y.m, z.m, s.data_ptr(), nbytes) == P.LF_OK
        only("y", y, rows=(r1,), cols=(n1,))
        only("z", z, rows=(r1,), cols=(n1,))
        return
    z, dy = matrix(rows, o, t, "z" in kept, normal(rows, o)), Framed(rows, o, t, normal(rows, o))
    dx, dw = Framed(rows, i, t) if what != "dw" else None, Framed(o, i, torch.float32) if what != "dx" else None
    db = torch.full((o,), MARK, device=DEV)
    spoil(x, r0, c1)
    w.t[n1, c0] = float("nan")
    dy.t[r1, n0] = float("nan")
    nbytes = P.lf_linear_backward_workspace_bytes(rows, o, i, dt)
    s = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
    assert P.lf_linear_backward(rows, o, i, dy.m, z.m, P.LF_ACT_SIGMOID, x.m if dw else None, w.m if dx else None, dx.m if dx else None,
                                dw.m if dw else None, db.data_ptr() if what == "backward" else 0, s.data_ptr(), nbytes) == P.LF_OK
    if dx:
        only("dx", dx, rows=(r1,), cols=(c0,))
    if dw:
        only("dw", dw, rows=(n0,), cols=(c1,))
    if what == "backward":
        assert db.isnan().nonzero().flatten().tolist() == [n0]
