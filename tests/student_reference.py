"""The student nets' operators in 64 bits on the CPU, for tests: from the definitions, with how far off arithmetic of 32 bits may be.

u = 2^-24 is half a step of fp32.  A sum of n terms in fp32, in any order, is off by at most n u times the sum of their magnitudes
(the square of u neglected); functions (division, square root, exponential, logarithm) count 8 u of their result and of their
argument's size.  Bounds are elementwise and leave the last rounding, to the result's type, to the caller."""
import math

import torch

U = 2.0 ** -24
BLOCK = 128
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


# ---- 8 bits with blocks of 128 --------------------------------------------------------------------------------------------
def least_exponent(top):
    """The least e >= -117 with top <= 448 * 2^e, element by element."""
    out = torch.full(top.shape, -117, dtype=torch.int64)
    for e in range(-117, 121):
        out += (top > 448 * 2.0 ** e).to(torch.int64)
    return out


def nearest_codes(v):
    """The e4m3 number nearest to each v (|v| <= 448), ties to the even significand."""
    a = v.abs()
    _, e = torch.frexp(a)                                     # a in [2^(e - 1), 2^e)
    step = torch.exp2((e.double() - 4).clamp(min=-9))         # 3 bits after the first; 2^-9 is the smallest number
    n = a / step
    low = torch.floor(n)
    up = (n - low > 0.5) | ((n - low == 0.5) & (low % 2 == 1))
    return torch.copysign((low + up) * step, v)


def pack(v):
    """(values of the codes, exponents [rows][groups]) of a matrix in 64 bits, groups of 128 along its rows.  What is not finite sets no scale
    and becomes NaN; a group of the largest scale holds at most 240 of it."""
    rows, cols = v.shape
    g = torch.nn.functional.pad(v, (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    finite = torch.where(torch.isfinite(g), g, 0.0)
    e = least_exponent(finite.abs().amax(-1))
    most = torch.where(e == 120, 240.0, 448.0).unsqueeze(-1)
    s = torch.maximum(torch.minimum(finite / torch.exp2(e.double()).unsqueeze(-1), most), -most)
    codes = torch.where(torch.isfinite(g), nearest_codes(s), math.nan)
    return codes.view(rows, -1)[:, :cols], e


def unpack(codes, e):
    return codes * torch.exp2(e.double()).repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def held(v):
    """What a matrix in 8 bits holds of v."""
    return unpack(*pack(v))


def pack_tiles(v):
    """The same with a scale for 128 x 128 values."""
    rows, cols = v.shape
    g = torch.nn.functional.pad(v, (0, -cols % BLOCK, 0, -rows % BLOCK))
    g = g.view(g.shape[0] // BLOCK, BLOCK, -1, BLOCK)
    finite = torch.where(torch.isfinite(g), g, 0.0)
    e = least_exponent(finite.abs().amax((1, 3)))
    wide = e[:, None, :, None]
    most = torch.where(wide == 120, 240.0, 448.0)
    s = torch.maximum(torch.minimum(finite / torch.exp2(wide.double()), most), -most)
    codes = torch.where(torch.isfinite(g), nearest_codes(s), math.nan)
    return codes.reshape(g.shape[0] * BLOCK, -1)[:rows, :cols], e


def held_tiles(v):
    codes, e = pack_tiles(v)
    scales = torch.exp2(e.double()).repeat_interleave(BLOCK, 0)[:v.shape[0]].repeat_interleave(BLOCK, 1)[:, :v.shape[1]]
    return codes * scales


# ---- layer norm -----------------------------------------------------------------------------------------------------------
def norm_forward(x, branch, gain, shift, eps):
    """{result: (value, bound)}"""
    s = x if branch is None else x + branch
    n = s.shape[1]
    mean = s.mean(1, keepdim=True)
    off = s - mean
    var = off.square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    y = off * rstd * gain + shift
    e_s = U * s.abs()
    e_mean = (n + 10) * U * s.abs().mean(1, keepdim=True)
    e_off = e_s + e_mean + U * off.abs()
    e_var = (2 * off.abs() * e_off + e_off.square()).mean(1, keepdim=True) + (n + 10) * U * (off.abs() + e_off).square().mean(1, keepdim=True)
    e_rstd = rstd * (0.5 * e_var / (var + eps) + 17 * U) * 1.01
    e_y = (off.abs() * e_rstd + rstd * e_off + 3 * U * off.abs() * rstd) * gain.abs() * 1.01 + U * y.abs() + U * shift.abs()
    return {"sum": (s, e_s * 0), "mean": (mean[:, 0], e_mean[:, 0]), "rstd": (rstd[:, 0], e_rstd[:, 0]), "y": (y, e_y)}


def norm_backward(dy, s, gain, mean, rstd, dsum):
    rows, n = s.shape
    rstd, mean = rstd[:, None], mean[:, None]
    h, t = (s - mean) * rstd, dy * gain
    by, level = (t * h).mean(1, keepdim=True), t.mean(1, keepdim=True)
    extra = torch.zeros_like(s) if dsum is None else dsum
    dx = extra + rstd * (t - level - h * by)
    e_by = (n + 16) * U * (t * h).abs().mean(1, keepdim=True)
    e_level = (n + 12) * U * t.abs().mean(1, keepdim=True)
    e_dx = rstd * (4 * U * (t.abs() + level.abs()) + e_level + h.abs() * (e_by + 6 * U * by.abs())) + 2 * U * ((t - level - h * by).abs() * rstd + extra.abs())
    dgain, dshift = (dy * h).sum(0), dy.sum(0)
    return {"dx": (dx, e_dx), "dgain": (dgain, (rows + 12) * U * (dy * h).abs().sum(0)), "dshift": (dshift, (rows + 8) * U * dy.abs().sum(0))}


# ---- products -------------------------------------------------------------------------------------------------------------
def _normal(z):
    return 0.5 * torch.erfc(-z / math.sqrt(2))


def act(z, name):
    sig = torch.sigmoid(z)
    return {"none": lambda: z, "sigmoid": lambda: sig, "relu": lambda: z.clamp(min=0), "silu": lambda: z * sig, "gelu": lambda: z * _normal(z)}[name]()


def slope(z, name):
    sig = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "sigmoid": lambda: sig * torch.sigmoid(-z), "relu": lambda: (z > 0).double(),
            "silu": lambda: sig * (1 + z * torch.sigmoid(-z)),
            "gelu": lambda: _normal(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[name]()


def product(x, w, exact):
    """x w^T of what both hold, and the bound.  exact: products are exact and summed in fp32.  Otherwise each eight consecutive products of a
    row are summed in 14 bits of their largest: every one may lose 2^-13 of it."""
    n = x.shape[1]
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    bound = (n + 40) * U * size
    if not exact:
        pad = -n % 8
        xs = torch.nn.functional.pad(x, (0, pad)).abs().view(x.shape[0], 1, -1, 8)
        ws = torch.nn.functional.pad(w, (0, pad)).abs().view(1, w.shape[0], -1, 8)
        for m in range(0, x.shape[0], 16):                    # (in parts: all products of a part are held)
            bound[m:m + 16] += 8 * 2.0 ** -13 * (xs[m:m + 16] * ws).amax(-1).sum(-1)
    return z, bound


def epilogue(z, e_z, bias, name, residual):
    """y and its bound from z = x w^T and its bound."""
    bias = torch.zeros(z.shape[1], dtype=torch.float64) if bias is None else bias
    v = z + bias
    e_v = e_z + U * v.abs()
    y = act(v, name)
    # no slope of an activation is above 1.13; values are functions of 8 u, of arguments up to v^2
    e_y = 1.13 * e_v + 16 * U * (y.abs() + (0 if name in ("none", "relu") else (v.abs() + v * v + 1) * torch.exp(-v.abs() / 2)))
    if residual is not None:
        y = y + residual
        e_y = e_y + U * y.abs()
    return (v, e_v), (y, e_y)


# ---- distillation ----------------------------------------------------------------------------------------------------------
def distil(z, t, classes, T, weight):
    """loss and gradient of each row with their bounds; t: minus infinity where there is no entry."""
    rows, n = z.shape
    there = classes >= 0
    t = torch.where(there, t, -math.inf)
    at = classes.clamp(min=0).long()
    most, top = z.amax(1, keepdim=True), t.amax(1, keepdim=True)
    x, y = (z - most) / T, (t - top) / T
    log_q, log_p = x - torch.log(torch.exp(x).sum(1, keepdim=True)), y - torch.log(torch.exp(y).sum(1, keepdim=True))
    q, p = torch.exp(log_q), torch.where(there, torch.exp(log_p), 0.0)
    # the exponential's argument is off by 4 u of it, the exponential by 2 u; sums by their number of terms; a division
    r_q, r_p = torch.where(q > 0, 4 * U * x.abs() + 2 * U, 0.0), torch.where(p > 0, 4 * U * y.abs() + 2 * U, 0.0)
    r_total, r_among = (q * r_q).sum(1, keepdim=True) + (n / 8 + 30) * U, (p * r_p).sum(1, keepdim=True) + (t.shape[1] + 8) * U
    gap = torch.where(p > 0, log_p - log_q.gather(1, at), 0.0)
    loss = (p * gap).sum(1)
    e_loss = (p * ((r_p + r_among + 2 * U) * gap.abs() + r_total + r_among)).sum(1) + U * loss.abs()
    d, e_d = q.clone(), q * (r_q + r_total + 4 * U) + 2.0 ** -126
    d.scatter_add_(1, at, -p)
    e_d.scatter_add_(1, at, p * (r_p + r_among + (t.shape[1] + 4) * U))
    e_d += 3 * U * d.abs()
    nothing = (weight == 0) | (top[:, 0] == -math.inf)
    scale = weight * T
    zero = torch.zeros(())
    return {"loss": (torch.where(nothing, zero, scale * T * loss), torch.where(nothing, zero, (scale * T).abs() * (e_loss + 2 * U * loss.abs()))),
            "dlogits": (torch.where(nothing[:, None], zero, scale[:, None] * d), torch.where(nothing[:, None], zero, scale[:, None].abs() * e_d))}
