"""Row-wise operators where a workgroup walks several rows, where sums over rows are joined, and where elements lie past 2^31; products
of matrices that long.  Against torch in 64 bits.

u = 2^-24 is half a step of fp32.  A row's sum is taken by threads of at most c = cols / 64 + 64 terms and a tree over them: off by at
most (c + 8) u of its magnitudes; a mean square in a root counts half of that, division and root 8 u each.  A sum over rows: (rows + 12) u."""
import pytest
import torch

import paper_1801_04928_amd as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def normal(t, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(shape))
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16).to(t)


def near(name, got, want, off):
    bound = off + (HALF[got.dtype] * (want.abs() + off)) + 1e-30
    assert bool(((got.double() - want).abs() <= bound).all()), name


def near_eight(name, m, rows, want, off):
    """Rows of a matrix in 8 bits."""
    part = P.E4M3Matrix.of(m.codes[rows], m.scales[rows], m.cols)
    scale = torch.exp2(part.scales.double() - 127).repeat_interleave(32, 1)[:, :m.cols]
    bound = off + torch.maximum(2.0 ** -4 * (want.abs() + off), 2.0 ** -10 * scale)
    assert bool(((part.load(dtype="f32").double() - want).abs() <= bound).all()), name


def norm_pass(rows, cols, dtype, kept, look):
    """A forward and a backward pass; the rows `look` and the gain's gradient are compared (the others' part of it by chunks)."""
    t = TYPE[dtype]
    n = P.RmsNorm(rows, cols, t, out="e4m3" if kept else t, eps=1e-5, device=DEV)
    n.gain.copy_(1 + normal(torch.float32, cols) / 8)
    x, branch, dy, dsum = normal(t, rows, cols), normal(t, rows, cols) / 2, normal(t, rows, cols) / 4, normal(t, rows, cols) / 8
    dy += 0.25
    y = n.forward(x, branch)
    stored = P.E4M3Matrix(rows, cols, device=DEV).save(n.sum) if kept else n.sum
    dx = n.backward(dy, dsum, stored=stored)
    gain, c = n.gain.double(), cols / 64 + 72
    s = x[look].double() + branch[look].double()
    rstd = (s.square().mean(1) + float(torch.tensor(1e-5))).rsqrt()
    off = (0.5 * c + 20) * U
    near("sum", n.sum[look], s, U * s.abs())
    near("rstd", n.rstd[look], rstd, off * rstd)
    want = s * rstd[:, None] * gain
    if kept:
        near_eight("y", y, look, want, (off + 8 * U) * want.abs())
        s = P.E4M3Matrix.of(stored.codes[look], stored.scales[look], cols).load(dtype="f32").double()
    else:
        near("y", y[look], want, (off + 8 * U) * want.abs())
        s = n.sum[look].double()
    r = n.rstd[look].double()[:, None]
    h, d = s * r, dy[look].double() * gain
    size = dsum[look].double().abs() + r * (d.abs() + h.abs() * (d * h).abs().mean(1, keepdim=True))
    near("dx", dx[look], dsum[look].double() + r * (d - h * (d * h).mean(1, keepdim=True)), (c + 8) * U * size)
    want, size = torch.zeros(cols, device=DEV, dtype=torch.float64), torch.zeros(cols, device=DEV, dtype=torch.float64)
    step = max(1, (1 << 26) // cols)
    for a in range(0, rows, step):
        part = slice(a, min(rows, a + step))
        s = P.E4M3Matrix.of(stored.codes[part], stored.scales[part], cols).load(dtype="f32") if kept else stored[part]
        dh = dy[part].double() * s.double() * n.rstd[part].double()[:, None]
        want += dh.sum(0)
        size += dh.abs().sum(0)
    near("dgain", n.dgain, want, (rows + 12) * U * size)


# more rows than workgroups, in every width that has kernels of its own; sums over rows of rows wider than what registers hold
@pytest.mark.parametrize("kept", [False, True], ids=["stored", "8bit"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(5000, 5), (2100, 65), (4500, 700), (600, 1500), (1100, 4100), (530, 8200), (17, 16400), (600, 20001),
                                   (1100, 17000)], ids=str)
def test_norm_of_many_rows(shape, dtype, kept):
    rows = shape[0]
    norm_pass(*shape, dtype, kept, slice(0, rows))


# more rows than a grid has workgroups; elements past 2^31
@pytest.mark.parametrize("kept", [False, True], ids=["stored", "8bit"])
@pytest.mark.parametrize("shape", [((1 << 22) + 2051, 12), ((1 << 20) + 1031, 2051)], ids=str)
def test_norm_of_very_many_rows(shape, kept):
    norm_pass(*shape, "bf16", kept, slice(shape[0] - 1500, shape[0]))


def test_8_bits_past_2_31_elements():
    rows, cols = (1 << 20) + 1031, 2051
    x = normal(torch.bfloat16, rows, cols)
    m = P.E4M3Matrix(rows, cols, device=DEV).save(x)
    back = m.load(dtype="bf16")
    for look in (slice(0, 300), slice(rows - 300, rows)):
        near_eight("8 bits", m, look, x[look].double(), torch.zeros((), device=DEV, dtype=torch.float64))
        part = P.E4M3Matrix(300, cols, device=DEV).save(x[look])
        assert torch.equal(part.codes, m.codes[look]) and torch.equal(part.scales, m.scales[look])
        assert torch.equal(back[look], part.load(dtype="bf16"))


@pytest.mark.parametrize("kept", [False, True], ids=["stored", "8bit"])
def test_product_past_2_31_elements(kept):
    """x and dx have 2.2e9 elements, and dw sums 270001 rows."""
    rows, o, i = 270001, 40, 8200
    x, w, dy = normal(torch.bfloat16, rows, i), normal(torch.bfloat16, o, i) / 64, normal(torch.bfloat16, rows, o)
    xk = P.E4M3Matrix(rows, i, device=DEV).save(x) if kept else x
    p = P.Linear(rows, o, i, "bf16", dw="f32", device=DEV)
    p.set_params(w)
    y = p.forward(xk)
    dx = p.backward(dy, xk)
    wide = w.double()
    for look in (slice(0, 300), slice(rows - 700, rows)):
        xv = (P.E4M3Matrix.of(xk.codes[look], xk.scales[look], i).load(dtype="f32") if kept else x[look]).double()
        near("y", y[look], torch.mm(xv, wide.t().contiguous()), (i + 8) * U * torch.mm(xv.abs(), wide.abs().t().contiguous()))
        d = dy[look].double()
        near("dx", dx[look], torch.mm(d, wide), (o + 8) * U * torch.mm(d.abs(), wide.abs()))
    want, size = torch.zeros(o, i, device=DEV, dtype=torch.float64), torch.zeros(o, i, device=DEV, dtype=torch.float64)
    for a in range(0, rows, 30000):
        part = slice(a, min(rows, a + 30000))
        xv = (P.E4M3Matrix.of(xk.codes[part], xk.scales[part], i).load(dtype="f32") if kept else x[part]).double()
        d = dy[part].double().t().contiguous()
        want += torch.mm(d, xv)
        size += torch.mm(d.abs(), xv.abs())
    near("dw", p.dw, want, (rows + 8) * U * size)
    near("db", p.db, dy.double().sum(0), (rows + 12) * U * dy.double().abs().sum(0))
