"""Matrices for the GPU tests of the student nets' operators: slices of larger ones, whose other elements are NaN where they are read and
a mark where they are written."""
import torch

import paper_1801_04928_amd as P
from tests import student_reference as R

DEV = "cuda:0"
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
MARK = 77.0


def values(seed, *shape, dtype="f32", std=1.0, mean=0.0):
    """Random values as the type holds them, in 64 bits on the CPU."""
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * std + mean).to(TYPE[dtype]).double()


class Dense:
    """`off` elements in front of every row, `pad` behind, a row above and below."""

    def __init__(self, rows, cols, dtype, values=None, off=0, pad=0):
        self.rows, self.cols, self.off = rows, cols, off
        fill = MARK if values is None else float("nan")
        self.all = torch.full((rows + 2, off + cols + pad), fill, dtype=TYPE[dtype], device=DEV)
        self.t = self.all[1:rows + 1, off:off + cols]
        if values is not None:
            self.t.copy_(values)
        self.m = P.lf_matrix(self.t.data_ptr() if rows else 0, self.all.shape[1], None, 0,
                             P.LF_MATRIX_F32 if dtype == "f32" else P.LF_MATRIX_BF16)

    def get(self):
        around = self.all.clone()
        around[1:self.rows + 1, self.off:self.off + self.cols] = MARK
        assert bool((around == MARK).all()), "written outside the matrix"
        return self.t.double().cpu()


class Blocks:
    """In 8 bits with blocks of 128; the codes past its last column are NaN where it is read, the scales past its last too."""

    def __init__(self, rows, cols, tiles=False, values=None, pad_groups=0):
        groups = -(-cols // 128)
        self.rows, self.cols, self.groups, self.tiles = rows, cols, groups, tiles
        self.scale_rows = -(-rows // 128) if tiles else rows
        self.codes = torch.full((rows + 1, (groups + pad_groups) * 128), 0x7f, dtype=torch.uint8, device=DEV)
        self.scales = torch.full((self.scale_rows + 1, -(-(groups + pad_groups) // 4) * 4), 255, dtype=torch.uint8, device=DEV)
        if values is not None:
            c, e = (R.pack_tiles if tiles else R.pack)(values)
            self.codes[:rows, :cols] = c.float().to(torch.float8_e4m3fn).view(torch.uint8).to(DEV)
            self.scales[:self.scale_rows, :groups] = (e + 127).to(torch.uint8).to(DEV)
        self.m = P.lf_matrix(self.codes.data_ptr(), self.codes.shape[1], self.scales.data_ptr(), self.scales.shape[1],
                             P.LF_MATRIX_E4M3_TILES if tiles else P.LF_MATRIX_E4M3_128)

    def raw(self):
        """(values of the codes, exponents), and that nothing around them was written."""
        codes, scales = self.codes.cpu(), self.scales.cpu()
        assert bool((codes[self.rows:] == 0x7f).all()) and bool((codes[:, self.groups * 128:] == 0x7f).all())
        assert bool((scales[self.scale_rows:] == 255).all())
        assert bool((codes[:self.rows, self.cols:self.groups * 128] == 0).all()), "codes past the last column are zero"
        return (codes[:self.rows, :self.cols].contiguous().view(torch.float8_e4m3fn).double(),
                scales[:self.scale_rows, :self.groups].to(torch.int64) - 127)


def same(name, got, want):
    """Equal, NaN where NaN are wanted."""
    assert got.shape == want.shape
    fine = (got == want) | (got.isnan() & want.isnan())
    assert bool(fine.all()), f"{name}: {int((~fine).sum())} of {fine.numel()} differ"


def near(name, got, want, bound):
    assert got.shape == want.shape, f"{name}: {got.shape} for {want.shape}"
    off = (got.double().cpu() - want).abs()
    assert bool(torch.isfinite(off).all()), f"{name}: not finite"
    if off.numel():
        at = int((off - bound).argmax())
        assert bool((off <= bound).all()), f"{name}[{at}]: {got.flatten()[at]} for {want.flatten()[at]}, {(bound + off * 0).flatten()[at]:.3g} allowed"


def near_rounded(name, got, want, bound):
    """A tensor whose values are known to `bound` before they are rounded to its type."""
    near(name, got, want, bound + R.HALF[got.dtype] * (want.abs() + bound) + 1e-40)


def near_blocks(name, m, want, bound):
    """A matrix in 8 bits (groups along its rows) whose values are known to `bound` before."""
    codes, e = m.raw()
    scale = torch.exp2(e.double())
    wide = scale.repeat_interleave(128, 1)[:, :want.shape[1]]
    near(name, R.unpack(codes, e), want, bound + torch.maximum(2.0 ** -4 * (want.abs() + bound), 2.0 ** -10 * wide))
    for g in range(e.shape[1]):                          # the least scale that holds the group, as far as it is known
        cols = slice(128 * g, 128 * g + 128)
        top, off = want[:, cols].abs().amax(1), bound[:, cols].amax(1)
        assert bool(((448 * scale[:, g] >= top - off) & ((224 * scale[:, g] < top + off) | (e[:, g] == -117))).all()), name
