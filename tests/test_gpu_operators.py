"""The residual blocks' operators on the GPU against the 64-bit reference.

Tolerances are worst cases of the arithmetic, elementwise: u = 2^-24 is half a step of fp32 and r half a step of the storage
type (0 for fp32, whose last rounding is among the u's; 2^-8 for bf16).  A sum of n terms in fp32, in any order, is off by at
most n u times the sum of their magnitudes (the square of u neglected).  Functions (division, square root, exp, erfc) are
counted as 8 u of their result and of their argument's size.  bf16 gradients have one more rounding, that of dz.
In 8 bits: codes are within half a step, 2^-4 of the value or 2^-10 of the scale.

Matrices are slices of larger ones, whose other elements are NaN where they are read and a mark where they are written."""
import numpy as np
import pytest
import torch

import paper_1801_04928_amd as P
from tests import operators_reference as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 0.0, "bf16": 2.0 ** -8}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
MARK = 77.0
DEV = "cuda:0"


def rounded(x, kind):
    """x as the storage type holds it, in 64 bits."""
    return torch.from_numpy(np.asarray(x)).to(TYPE[kind]).double().numpy()


class Dense:
    """A matrix inside a larger one: `off` elements in front of every row, `pad` behind."""

    def __init__(self, rows, cols, kind, values=None, off=0, pad=0):
        self.rows, self.cols, self.off = rows, cols, off
        fill = MARK if values is None else float("nan")
        self.all = torch.full((rows + 2, off + cols + pad), fill, dtype=TYPE[kind], device=DEV)
        self.t = self.all[1:rows + 1, off:off + cols]
        if values is not None:
            self.t.copy_(torch.from_numpy(np.asarray(values)))
        self.m = P.lf_matrix(self.t.data_ptr() if rows else 0, self.all.shape[1], None, 0,
                             P.LF_MATRIX_F32 if kind == "f32" else P.LF_MATRIX_BF16)

    def get(self):
        """The values, and that nothing around them was written."""
        around = self.all.clone()
        around[1:self.rows + 1, self.off:self.off + self.cols] = MARK
        assert bool((around == MARK).all()), "written outside the matrix"
        return self.t.double().cpu().numpy()


class Eight:
    """A matrix in 8 bits inside a larger one; the codes past its last column are NaN where it is read."""

    def __init__(self, rows, cols, values=None, pad_groups=0):
        groups = -(-cols // 32)
        self.rows, self.cols, self.groups = rows, cols, groups
        self.codes = torch.full((rows + 1, (groups + pad_groups) * 32), 0x7f, dtype=torch.uint8, device=DEV)
        self.scales = torch.full((rows + 1, groups + pad_groups + 3), 200, dtype=torch.uint8, device=DEV)
        if values is not None:
            c, s = R.to_eight(values)
            self.codes[:rows, :cols] = torch.from_numpy(c).to(DEV)
            self.scales[:rows, :groups] = torch.from_numpy(s).to(DEV)
        self.m = P.lf_matrix(self.codes.data_ptr(), self.codes.shape[1], self.scales.data_ptr(), self.scales.shape[1],
                             P.LF_MATRIX_E4M3)

    def raw(self):
        codes, scales = self.codes.cpu().numpy(), self.scales.cpu().numpy()
        assert (codes[self.rows:] == 0x7f).all() and (codes[:, self.groups * 32:] == 0x7f).all()
        assert (scales[self.rows:] == 200).all() and (scales[:, self.groups:] == 200).all()
        assert (codes[:self.rows, self.cols:self.groups * 32] == 0).all(), "codes past the last column are zero"
        return codes[:self.rows, :self.cols], scales[:self.rows, :self.groups]

    def get(self):
        return R.from_eight(*self.raw())


def matrix(rows, cols, kind, dtype, values=None, off=0, pad=0):
    if kind == "e4m3":
        return Eight(rows, cols, values, pad_groups=1 if pad else 0)
    return Dense(rows, cols, dtype, values, off, pad)


def held(values, kind, dtype):
    """What a matrix holds of values."""
    return R.from_eight(*R.to_eight(rounded(values, dtype))) if kind == "e4m3" else rounded(values, dtype)


def near(name, got, want, bound):
    off = np.abs(got - want)
    assert got.shape == want.shape and np.isfinite(got).all(), f"{name}: not finite"
    worst = np.unravel_index(np.argmax(off - bound), off.shape) if off.size else None
    fine = off.size == 0 or bool((off <= bound).all())
    assert fine, f"{name}{list(worst)}: {got[worst]} for {want[worst]}, {bound[worst]:.3g} allowed"


def near_kept(name, m, want, bound, dtype):
    """m holds `want`, known to `bound`, in its type."""
    if isinstance(m, Dense):
        near(name, m.get(), want, bound + HALF[dtype] * (np.abs(want) + bound))
        return
    codes, scales = m.raw()
    got = R.from_eight(codes, scales)
    exponent = np.repeat(scales.astype(np.int64) - 127, 32, axis=1)[:, :want.shape[1]]
    near(name, got, want, bound + np.maximum(2.0 ** -4 * (np.abs(want) + bound), 2.0 ** -10 * 2.0 ** exponent))
    for g in range(scales.shape[1]):                    # the least scale that holds the group, as far as it is known
        cols = slice(32 * g, 32 * g + 32)
        top, off = np.abs(want[:, cols]).max(1), bound[:, cols].max(1)
        e = scales[:, g].astype(np.int64) - 127
        assert (448 * 2.0 ** e >= top - off).all() and ((448 * 2.0 ** (e - 1) < top + off) | (e == -117)).all(), name


def call(status):
    assert status == P.LF_OK, P.lf_operator_error()


def sync():
    torch.cuda.synchronize()


# ---- 8 bits ----------------------------------------------------------------------------------------------------------
SHAPES = [(0, 5), (1, 1), (1, 32), (3, 31), (2, 33), (5, 40), (4, 64), (7, 100), (70, 257), (300, 72), (9, 1111), (3, 8200), (2, 20000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_checkpoint_is_exact(rows, cols, dtype):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=(rows, cols)) * 3) * 10.0 ** rng.integers(-30, 30, size=(rows, 1))
    x = rounded(x, dtype)
    source, kept = Dense(rows, cols, dtype, x, off=1, pad=2), Eight(rows, cols, pad_groups=1)
    call(P.lf_checkpoint_save(rows, cols, source.m, kept.m))
    sync()
    codes, scales = kept.raw()
    want_codes, want_scales = R.to_eight(x)
    assert np.array_equal(scales, want_scales) and np.array_equal(codes, want_codes)
    back = Dense(rows, cols, dtype, off=3, pad=1)
    call(P.lf_checkpoint_load(rows, cols, kept.m, back.m))
    sync()
    assert np.array_equal(back.get(), R.from_eight(codes, scales))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_checkpoint_of_what_is_not_ordinary(dtype):
    """NaN, infinities, zeros of both signs, the largest and the smallest numbers, ties, groups of nothing else."""
    t = TYPE[dtype]
    big, tiny = torch.finfo(t).max, torch.finfo(t).tiny
    x = np.zeros((12, 64))
    x[0, 0], x[0, 5], x[0, 40] = np.nan, 3.0, np.inf
    x[1] = np.nan
    x[2, ::2], x[2, 1::2] = np.inf, -np.inf
    x[3, 0], x[3, 1], x[3, 2] = big, -big, 1.0
    x[4, 0], x[4, 40] = tiny, -tiny / 4
    x[5, 3], x[5, 4] = -0.0, 448.0
    x[6, :17] = np.concatenate([[448.0], 17 + np.arange(16) * 2.0])     # ties between codes of 16..32 lie at the odd numbers
    x[7, 0], x[7, 1] = 448.0, 2.0 ** -10                                  # half of the smallest code: to even, zero
    x[8, 0], x[8, 1] = 448.0, 1.5 * 2.0 ** -9
    x[9, 0] = 1.75 * 2.0 ** 127 if dtype == "f32" else 1.75 * 2.0 ** 126
    x[10, 0], x[10, 1] = 450.0, 1.0
    x[11, 33] = tiny * 2.0 ** 10
    x = rounded(x, dtype)
    source, kept = Dense(12, 64, dtype, x), Eight(12, 64)
    call(P.lf_checkpoint_save(12, 64, source.m, kept.m))
    sync()
    codes, scales = kept.raw()
    want_codes, want_scales = R.to_eight(x)
    assert np.array_equal(scales, want_scales)
    nan = np.isnan(R.TABLE[want_codes])
    assert np.array_equal(np.isnan(R.TABLE[codes]), nan) and np.array_equal(codes[~nan], want_codes[~nan])
    for out in ("f32", "bf16"):
        back = Dense(12, 64, out)
        call(P.lf_checkpoint_load(12, 64, kept.m, back.m))
        sync()
        got, want = back.get(), R.from_eight(codes, scales)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~nan], want[~nan])
        assert np.isfinite(got[3]).all()


# ---- norm ------------------------------------------------------------------------------------------------------------
NORMS = [(0, 5), (1, 1), (1, 7), (2, 8), (3, 33), (5, 511), (6, 512), (9, 513), (4, 1024), (7, 1500), (5, 2048), (3, 2049), (2, 4100),
         (3, 8192), (2, 8200), (2, 16384), (2, 16385), (3, 20001), (700, 65)]


def sum_error(n):
    return (n + 8) * U


@pytest.mark.parametrize("dtype, out", [("f32", "f32"), ("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("rows, cols", NORMS)
def test_norm_forward(rows, cols, dtype, out):
    rng = np.random.default_rng(cols)
    with_branch, with_gain, with_sum = cols % 2 == 0, cols % 3 != 0, rows != 3
    x = rounded(rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=cols)), dtype)
    branch = rounded(rng.normal(size=(rows, cols)), dtype) if with_branch else None
    gain = rounded(1 + 0.2 * rng.normal(size=cols), "f32")
    eps = 1e-5
    mx, my = Dense(rows, cols, dtype, x, off=1, pad=1), matrix(rows, cols, out, dtype, pad=3)
    mb = Dense(rows, cols, dtype, branch, off=2, pad=5) if with_branch else None
    ms = Dense(rows, cols, dtype, off=5, pad=3) if with_sum else None
    g = torch.from_numpy(gain).float().to(DEV)
    rstd = torch.full((rows + 1,), MARK, device=DEV)
    call(P.lf_norm_forward(rows, cols, mx.m, mb.m if mb else None, g.data_ptr() if with_gain else 0, eps, ms.m if ms else None,
                           my.m, rstd.data_ptr()))
    sync()
    s, want_rstd, y = R.norm_forward(x, branch, gain if with_gain else np.ones(cols), np.float32(eps).astype(np.float64))
    # (a thread adds up at most cols / 64 + 64 squares, then a tree of its neighbours' sums)
    rel = 0.5 * sum_error(cols / 64 + 64) + 16 * U + 2 * U
    got = rstd.double().cpu().numpy()
    assert got[rows] == MARK
    near("rstd", got[:rows], want_rstd, rel * want_rstd)
    if ms:
        near_kept("sum", ms, s, U * np.abs(s), dtype)
    near_kept("y", my, y, (rel + 4 * U) * np.abs(y) + 2 * U * np.abs(y), dtype)


def test_norm_of_rows_without_anything():
    """A row of zeros, with eps and without; a row with a NaN or an infinity spoils itself alone."""
    x = np.ones((4, 48))
    x[0], x[1, 3], x[2, 40] = 0.0, np.nan, np.inf
    for out in ("bf16", "e4m3"):
        for eps in (1e-6, 0.0):
            mx, my, rstd = Dense(4, 48, "bf16", x), matrix(4, 48, out, "bf16"), torch.empty(4, device=DEV)
            call(P.lf_norm_forward(4, 48, mx.m, None, 0, eps, None, my.m, rstd.data_ptr()))
            sync()
            y = my.get()
            assert (y[0] == 0).all() if eps else np.isnan(y[0]).all()
            assert np.isnan(y[1]).all() and np.isnan(y[2, 40]) and (np.delete(y[2], 40) == 0).all()
            assert np.abs(y[3] - 1).max() < 2.0 ** -7


@pytest.mark.parametrize("cols", [40, 700, 20000])
def test_norm_sum_in_place(cols):
    rng = np.random.default_rng(3)
    x, branch = rounded(rng.normal(size=(5, cols)), "bf16"), rounded(rng.normal(size=(5, cols)), "bf16")
    apart = [Dense(5, cols, "bf16", x), Dense(5, cols, "bf16", branch), Dense(5, cols, "bf16"), Eight(5, cols)]
    call(P.lf_norm_forward(5, cols, apart[0].m, apart[1].m, 0, 1e-6, apart[2].m, apart[3].m, 0))
    for which in (0, 1):
        both = [Dense(5, cols, "bf16", x), Dense(5, cols, "bf16", branch)]
        y = Eight(5, cols)
        call(P.lf_norm_forward(5, cols, both[0].m, both[1].m, 0, 1e-6, both[which].m, y.m, 0))
        sync()
        assert torch.equal(both[which].t, apart[2].t) and torch.equal(y.codes, apart[3].codes)
        assert torch.equal(y.scales, apart[3].scales)


@pytest.mark.parametrize("dtype, stored", [("f32", "f32"), ("f32", "e4m3"), ("bf16", "bf16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("rows, cols", NORMS)
def test_norm_backward(rows, cols, dtype, stored):
    rng = np.random.default_rng(cols + 1)
    with_dsum, with_gain, with_dgain = cols % 2 == 1, cols % 3 != 0, rows != 2
    total = held(rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=cols)), stored, dtype)
    dy = rounded(rng.normal(size=(rows, cols)), dtype)
    dsum = rounded(rng.normal(size=(rows, cols)), dtype) if with_dsum else None
    gain = rounded(1 + 0.2 * rng.normal(size=cols), "f32") if with_gain else np.ones(cols)
    rstd = rounded(1 / np.sqrt((total * total).mean(1) + 1e-5), "f32")
    mdy, ms = Dense(rows, cols, dtype, dy, off=1), matrix(rows, cols, stored, dtype, total, off=2, pad=1)
    mds = Dense(rows, cols, dtype, dsum, pad=3) if with_dsum else None
    mdx = Dense(rows, cols, dtype, off=3)
    g, r = torch.from_numpy(gain).float().to(DEV), torch.from_numpy(rstd).float().to(DEV)
    dgain = torch.full((cols + 1,), MARK, device=DEV)
    nbytes = P.lf_norm_workspace_bytes(rows, cols)
    scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
    call(P.lf_norm_backward(rows, cols, mdy.m, ms.m, g.data_ptr() if with_gain else 0, r.data_ptr(), mds.m if mds else None, mdx.m,
                            dgain.data_ptr() if with_dgain else 0, scratch.data_ptr(), nbytes))
    sync()
    assert bool((scratch[nbytes:] == 255).all())
    want, want_gain = R.norm_backward(dy, total, gain, rstd, dsum)
    h, t = np.abs(total * rstd[:, None]), np.abs(dy * gain)
    size = rstd[:, None] * (t + h * (t * h).mean(1, keepdims=True)) + (0 if dsum is None else np.abs(dsum))
    near_kept("dx", mdx, want, (sum_error(cols / 64 + 64) + 8 * U) * size, dtype)
    got = dgain.double().cpu().numpy()
    assert got[cols] == MARK
    if with_dgain:
        near("dgain", got[:cols], want_gain, sum_error(rows + 4) * (np.abs(dy) * h).sum(0))
    else:
        assert (got == MARK).all()


# ---- product -----------------------------------------------------------------------------------------------------------
# rows, outputs, inputs: single samples, few rows, sizes around every tile's, contractions that are split and ragged ones
PRODUCTS = [(0, 9, 7), (1, 1, 1), (1, 64, 200), (1, 1000, 1027), (2, 33, 8), (7, 100, 65), (16, 48, 640), (17, 31, 63), (31, 129, 64),
            (33, 32, 515), (64, 64, 128), (65, 65, 129), (100, 257, 72), (128, 256, 2048), (130, 40, 4100), (257, 300, 333),
            (300, 1030, 96), (1100, 1540, 70), (513, 1025, 264)]
ACTS = ["none", "sigmoid", "relu", "silu", "gelu"]


def small(rng, dtype, *shape):
    return rounded(rng.normal(size=shape), dtype)


def scratch_of(nbytes):
    s = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
    return s, nbytes


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", PRODUCTS, ids=str)
def test_linear_forward(shape, dtype):
    rows, o, i = shape
    for turn, (x_kind, y_kind, z_kind) in enumerate([("same", "same", "none"), ("same", "e4m3", "same"), ("e4m3", "same", "e4m3"),
                                                     ("e4m3", "e4m3", "none")]):
        rng = np.random.default_rng(rows + 7 * o + 31 * i + turn)
        act = ACTS[(rows + o + turn) % 5]
        x = held(rng.normal(size=(rows, i)), x_kind, dtype)
        w, bias = small(rng, dtype, o, i) * i ** -0.5, rounded(rng.normal(size=o), "f32") if turn != 1 else None
        w = rounded(w, dtype)
        residual = small(rng, dtype, rows, o) if turn % 2 == 0 else None
        # aligned rows in one turn, odd ones in the others
        p = [0, 1, 3, 8][turn]
        mx, mw = matrix(rows, i, x_kind, dtype, x, off=p, pad=p), Dense(o, i, dtype, w, off=p, pad=-i % 8 if turn == 0 else p)
        mr = Dense(rows, o, dtype, residual, off=1) if residual is not None else None
        my, mz = matrix(rows, o, y_kind, dtype, off=p, pad=2), matrix(rows, o, z_kind, dtype, off=1) if z_kind != "none" else None
        b = torch.from_numpy(bias).float().to(DEV) if bias is not None else None
        s, nbytes = scratch_of(P.lf_linear_workspace_bytes(rows, o, i, P.LF_F32 if dtype == "f32" else P.LF_BF16))
        call(P.lf_linear_forward(rows, o, i, mx.m, mw.m, b.data_ptr() if b is not None else 0, P.operators.ACTIVATIONS[act],
                                 mr.m if mr else None, my.m, mz.m if mz else None, s.data_ptr(), nbytes))
        sync()
        assert bool((s[nbytes:] == 255).all())
        z, y = R.linear_forward(x, w, bias, act, residual)
        size = np.abs(x) @ np.abs(w).T + (0 if bias is None else np.abs(bias))
        z_off = sum_error(i) * size
        if mz:
            near_kept(f"z of turn {turn}", mz, z, z_off, dtype)
        # no activation's slope is above 1.13
        y_off = 1.13 * z_off + 16 * U * np.maximum(np.abs(z), 1) + 2 * U * (np.abs(y) + (0 if residual is None else np.abs(residual)))
        near_kept(f"y of turn {turn}, {act}", my, y, y_off, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", PRODUCTS, ids=str)
def test_linear_backward(shape, dtype):
    rows, o, i = shape
    for turn, (x_kind, z_kind, dw_kind) in enumerate([("same", "same", "same"), ("same", "e4m3", "f32"), ("e4m3", "same", "f32"),
                                                      ("e4m3", "e4m3", "same")]):
        rng = np.random.default_rng(rows + 5 * o + 17 * i + turn)
        act = ACTS[(rows + i + turn) % 5]
        x, z = held(rng.normal(size=(rows, i)), x_kind, dtype), held(rng.normal(size=(rows, o)), z_kind, dtype)
        w, dy = rounded(small(rng, dtype, o, i) * i ** -0.5, dtype), small(rng, dtype, rows, o)
        want_dx, want_dw, want_db = [(True, True, True), (True, True, False), (False, True, True), (True, False, False)][turn]
        p = [0, 1, 3, 8][turn]
        mx, mz = matrix(rows, i, x_kind, dtype, x, off=p, pad=p), matrix(rows, o, z_kind, dtype, z, off=1)
        mw, mdy = Dense(o, i, dtype, w, off=p, pad=-i % 8 if turn == 0 else p), Dense(rows, o, dtype, dy, off=p, pad=1)
        mdx, mdw = Dense(rows, i, dtype, off=p, pad=p), Dense(o, i, "f32" if dw_kind == "f32" else dtype, off=1)
        db = torch.full((o + 1,), MARK, device=DEV)
        s, nbytes = scratch_of(P.lf_linear_backward_workspace_bytes(rows, o, i, P.LF_F32 if dtype == "f32" else P.LF_BF16))
        call(P.lf_linear_backward(rows, o, i, mdy.m, mz.m if act != "none" else None, P.operators.ACTIVATIONS[act],
                                  mx.m if want_dw else None, mw.m if want_dx else None, mdx.m if want_dx else None,
                                  mdw.m if want_dw else None, db.data_ptr() if want_db else 0, s.data_ptr(), nbytes))
        sync()
        assert bool((s[nbytes:] == 255).all())
        dz, dx, dw, dbias = R.linear_backward(dy, z, act, x, w)
        # slopes are sums of products of functions: 24 u of the sizes in them
        before = np.abs(dy) * (24 * U * (1 + np.abs(z)) if act != "none" else 0)
        dz_off = before + (HALF[dtype] * (np.abs(dz) + before) if act != "none" else 0)
        if want_dx:
            near_kept(f"dx of turn {turn}, {act}", mdx, dx, dz_off @ np.abs(w) + sum_error(o) * ((np.abs(dz) + dz_off) @ np.abs(w)), dtype)
        else:
            assert (mdx.get() == MARK).all()
        if want_dw:
            bound = dz_off.T @ np.abs(x) + sum_error(rows) * ((np.abs(dz) + dz_off).T @ np.abs(x))
            near_kept(f"dw of turn {turn}, {act}", mdw, dw, bound, "f32" if dw_kind == "f32" else dtype)
        else:
            assert (mdw.get() == MARK).all()
        got = db.double().cpu().numpy()
        assert got[o] == MARK
        if want_db:
            near(f"db of turn {turn}", got[:o], dbias, before.sum(0) + sum_error(rows + 4) * np.abs(dz).sum(0))
        else:
            assert (got[:o] == MARK).all()


# Sizes that the tiles of 256 and 128 take, with ends in every direction and rows at odd addresses; a contraction split over
# workgroups; up to four rows; one row of tiles more than the compute units take at once.
LARGE = [(4090, 4083, 203), (4096, 4104, 136), (2050, 2040, 520), (1030, 1000, 4200), (3, 515, 1100), (4, 4097, 777), (2, 100, 5),
         (260, 8200, 328)]


def oracle_product(p, q):
    """p q^T in 64 bits on the GPU, of operands laid out whole."""
    return torch.mm(p.double().contiguous(), q.double().t().contiguous())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kept", [False, True], ids=["stored", "8bit"])
@pytest.mark.parametrize("shape", LARGE, ids=str)
def test_linear_large(shape, kept, dtype):
    rows, o, i = shape
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + o + i)

    def normal(*size, std=1.0):
        return (torch.randn(*size, generator=g, device=DEV) * std).to(t)

    # rows one element longer than what is used: no row but the first begins at a multiple of 16 bytes
    x, w, dy = normal(rows, i + 1)[:, :i], normal(o, i + 1, std=i ** -0.5)[:, :i], normal(rows, o + 1)[:, :o]
    bias, residual = normal(o).float(), normal(rows, o)
    xk = P.E4M3Matrix(rows, i, device=DEV).save(x) if kept else x
    xv = xk.load(dtype="f32") if kept else x.float()
    p = P.Linear(rows, o, i, dtype, act="relu", z="e4m3" if kept else dtype, dw="f32", device=DEV)
    p.set_params(w, bias)
    y = p.forward(xk, residual)
    z = oracle_product(xv, w) + bias.double()
    size = oracle_product(xv.abs(), w.abs()) + bias.abs()
    z_off = sum_error(i) * size
    want = z.clamp(min=0) + residual.double()
    y_off = z_off + U * (z.abs() + want.abs()) + HALF[dtype] * (want.abs() + z_off) + 1e-30
    assert bool(((y.double() - want).abs() <= y_off).all())
    zv = p.z.load(dtype="f32").double() if kept else p.z.double()
    sign = zv > 0
    dx = p.backward(dy, xk)
    dz = torch.where(sign, dy.double(), 0.0)
    for name, got, a, b, n, half in [("dx", dx, dz, w.t(), o, HALF[dtype]), ("dw", p.dw, dz.t(), xv.t(), rows, U)]:
        want, size = oracle_product(a, b), oracle_product(a.abs(), b.abs())
        off = sum_error(n) * size
        assert bool(((got.double() - want).abs() <= off + half * (want.abs() + off) + 1e-30).all()), name
    off = sum_error(rows) * dz.abs().sum(0) + 1e-30
    assert bool(((p.db.double() - dz.sum(0)).abs() <= off).all())


@pytest.mark.parametrize("act", ACTS)
def test_activations_far_out(act):
    """Arguments from the smallest to the largest: y and the gradient before the activation, at single elements (inputs = 1)."""
    z = np.concatenate([[0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3], np.linspace(-20, 20, 401), [-87.0, 87.0, -89.0, 89.0, -104.0, 104.0, 1e4, -1e4,
                        1e30, -1e30]]).astype(np.float32).astype(np.float64)
    n = len(z)
    mx, one = Dense(n, 1, "f32", z[:, None]), Dense(1, 1, "f32", np.ones((1, 1)))
    y = Dense(n, 1, "f32")
    a = P.operators.ACTIVATIONS[act]
    call(P.lf_linear_forward(n, 1, 1, mx.m, one.m, 0, a, None, y.m, None, 0, 0))
    dx, dy = Dense(n, 1, "f32"), Dense(n, 1, "f32", np.ones((n, 1)))
    s, nbytes = scratch_of(P.lf_linear_backward_workspace_bytes(n, 1, 1, P.LF_F32))
    call(P.lf_linear_backward(n, 1, 1, dy.m, mx.m, a, None, one.m, dx.m, None, 0, s.data_ptr(), nbytes))
    sync()
    near("y", y.get()[:, 0], R.act(z, act), 16 * U * np.minimum(np.maximum(np.abs(z), 1), 1e38) * (np.abs(R.act(z, act)) > 0) + 1e-37
         + 16 * U * np.abs(R.act(z, act)))
    near("slope", dx.get()[:, 0], R.slope(z, act), 24 * U * (1 + np.minimum(np.abs(z), 30)))


def test_spoiled_rows_stay_alone():
    """A NaN in a row of x, or of dy, reaches that row's results and (dw, db) those its column sums are part of, no others."""
    rng = np.random.default_rng(9)
    for kind in ("same", "e4m3"):
        x = held(rng.normal(size=(70, 96)), kind, "bf16")
        mx = matrix(70, 96, kind, "bf16", x)
        if kind == "e4m3":
            mx.codes[13, 5] = 0x7f
        else:
            mx.t[13, 5] = float("nan")
        w, y = Dense(80, 96, "bf16", small(rng, "bf16", 80, 96)), Dense(70, 80, "bf16")
        call(P.lf_linear_forward(70, 80, 96, mx.m, w.m, 0, P.LF_ACT_RELU, None, y.m, None, 0, 0))
        dy, dw, dx = Dense(70, 80, "bf16", small(rng, "bf16", 70, 80)), Dense(80, 96, "f32"), Dense(70, 96, "bf16")
        dy.t[21, 7] = float("nan")
        s, nbytes = scratch_of(P.lf_linear_backward_workspace_bytes(70, 80, 96, P.LF_BF16))
        db = torch.empty(80, device=DEV)
        call(P.lf_linear_backward(70, 80, 96, dy.m, None, P.LF_ACT_NONE, mx.m, w.m, dx.m, dw.m, db.data_ptr(), s.data_ptr(), nbytes))
        sync()
        bad = np.isnan(y.get())
        assert bad[13].all() and bad.sum() == 80
        bad = np.isnan(dx.get())
        assert bad[21].all() and bad.sum() == 96
        bad = np.isnan(dw.get())
        assert bad[7].all() and bad[:, 5].all() and bad.sum() == 96 + 80 - 1
        assert torch.isnan(db).nonzero().flatten().tolist() == [7]


# ---- objects, graphs, streams --------------------------------------------------------------------------------------------
def block_pass(net, x, dy):
    y = net.forward(x)
    return [y, net.backward(dy), *net.dw1, *net.dw2, *net.db1, *net.db2, *net.dgain]


def make_net(rows, dtype="bf16", checkpoints="e4m3", depth=2, width=72, hidden=136, act="gelu"):
    net = P.ResidualNet(depth, width, hidden, rows, dtype=dtype, act=act, checkpoints=checkpoints)
    net.init(3)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    for v in [*net.b1, *net.b2]:
        v.copy_(torch.randn(v.shape, generator=g, device=DEV) * 0.1)
    x = torch.randn(rows, width, generator=g, device=DEV).to(net.dtype)
    return net, x, torch.randn(rows, width, generator=g, device=DEV).to(net.dtype)


def test_fewer_rows_and_the_same_bits():
    """An object made for more rows gives a smaller call's results, twice the same bits."""
    net, x, dy = make_net(200)
    few, _, _ = make_net(37)
    want = [v.clone() for v in block_pass(few, x[:37], dy[:37])]
    for _ in range(2):
        got = block_pass(net, x[:37], dy[:37])
        sync()
        assert got[0].shape == (37, 72)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("checkpoints", ["e4m3", "bf16"])
def test_net_in_a_graph_and_on_another_stream(checkpoints):
    net, x, dy = make_net(130, checkpoints=checkpoints)
    eager = [v.clone() for v in block_pass(net, x, dy)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = block_pass(net, x, dy)
    side.synchronize()
    for a, b in zip(other, eager):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block_pass(net, x, dy)
    for turn in range(3):
        x2 = x * (turn + 1) / 2
        for v in out:
            v.zero_()
        kept = x.clone()
        x.copy_(x2)
        graph.replay()
        sync()
        got = [v.clone() for v in out]
        want = [v.clone() for v in block_pass(net, x, dy)]
        sync()
        x.copy_(kept)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("act", ["gelu", "silu", "sigmoid", "none"])
def test_net_is_the_reference_chain(act):
    """fp32, nothing in 8 bits: output and all gradients against the blocks' formulas in 64 bits."""
    net, x, dy = make_net(45, "f32", "f32", act=act)
    got = [v.double().cpu().numpy() for v in block_pass(net, x, dy)]
    sync()
    as64 = lambda vs: [v.double().cpu().numpy() for v in vs]     # noqa: E731
    w1, w2, b1, b2, gain = map(as64, (net.w1, net.w2, net.b1, net.b2, net.gain))
    s, branch, kept = x.double().cpu().numpy(), None, []
    for b in range(2):
        s, rstd, h = R.norm_forward(s, branch, gain[b], np.float64(np.float32(1e-6)))
        z, u = R.linear_forward(h, w1[b], b1[b], act, None)
        _, branch = R.linear_forward(u, w2[b], b2[b], "none", None)
        kept.append((s, rstd, h, z, u))
    ds, grads = dy.double().cpu().numpy(), [None, None]
    for b in (1, 0):
        s0, rstd, h, z, u = kept[b]
        _, du, dw2, db2 = R.linear_backward(ds, None, "none", u, w2[b])
        _, dh, dw1, db1 = R.linear_backward(du, z, act, h, w1[b])
        ds, dgain = R.norm_backward(dh, s0, gain[b], rstd, ds)
        grads[b] = (dw1, dw2, db1, db2, dgain)
    want = [s + branch, ds] + [grads[b][k] for k in range(5) for b in range(2)]
    for k, (a, b) in enumerate(zip(got, want)):
        # normwise: a chain of six products of at most 136 terms
        assert np.linalg.norm(a - b) <= 6 * 150 * U * np.linalg.norm(b) + 1e-12, k


def test_training_with_8_bit_activations_lowers_the_cost():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_residual_net.py")
    spec = importlib.util.spec_from_file_location("train_residual_net", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    costs = {}
    for checkpoints in ("e4m3", "f32"):
        first, last, _, _ = example.train(depth=2, width=64, hidden=128, rows=128, steps=60, checkpoints=checkpoints, say=lambda *a, **k: None)
        costs[checkpoints] = last
        assert last < 0.7 * first
    assert costs["e4m3"] < 1.1 * costs["f32"]


def test_objects_refuse():
    n = P.RmsNorm(4, 40, "bf16", passes="forward")
    x = torch.zeros(5, 40, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(P.LfError, match="5 rows"):
        n.forward(x)
    with pytest.raises(P.LfError, match="x: 4 x 40"):
        n.forward(torch.zeros(4, 40, dtype=torch.bfloat16))
    with pytest.raises(P.LfError, match="type"):
        n.forward(x[:4].float())
    with pytest.raises(P.LfError, match="backward"):
        n.backward(x[:4])
