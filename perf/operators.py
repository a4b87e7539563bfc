"""The operators of residual blocks, as cases that can be prepared, run and timed: the root-mean-square norm with the
residual's addition, the matrix product with bias, activation and residual in its epilogue, both with their backward
passes, and activations kept in 8 bits, which the norm and the product write and the backward passes read.

`run` computes an operator in its plain form (`own` false: elementary torch operations in 32 bits, rounded once at the
end) or through this package's entry points (`own` true).  `exact` computes the same from the definition in 64 bits.

8 bits: e4m3 codes with one power-of-two scale (e8m0) per group of 32 columns of a row; rows of codes are padded to whole
groups.  A matrix in 8 bits comes back as its codes and its scales, in the float types that stand for their values.

Shapes: rows x cols for norms and checkpoints; rows x inputs times (outputs x inputs)^T for products.  The ranges: 1 to
16384 rows (one sample to a long minibatch), 8 to 16384 columns, products of 16 to 8192 inputs and outputs, with sizes that
are no multiple of anything among them."""
import math

import torch

own = False

GROUP = 32
LOWEST = -117                       # the smallest scale: 2^-117 times the smallest code is a normal bf16 number
ELEMENTS = 16384 * 8192             # the largest norm or checkpoint
FLOPS = 2 * 4096 * 8192 * 8192      # the largest single product (a backward pass is two of them)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DEVICE = "cuda:0"
EPS = 1e-6


def _norm(name, rows, cols, dtype, out):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "out": out}


def _norm_back(name, rows, cols, dtype, stored):
    return {"name": name, "op": "norm_back", "rows": rows, "cols": cols, "dtype": dtype, "stored": stored}


def _product(name, rows, outputs, inputs, dtype, act, x, y, z, residual):
    return {"name": name, "op": "product", "rows": rows, "outputs": outputs, "inputs": inputs, "dtype": dtype,
            "act": act, "x": x, "y": y, "z": z, "residual": residual}


def _product_back(name, rows, outputs, inputs, dtype, act, x, z):
    return {"name": name, "op": "product_back", "rows": rows, "outputs": outputs, "inputs": inputs, "dtype": dtype,
            "act": act, "x": x, "z": z}


def _checkpoint(name, rows, cols, dtype):
    return {"name": name, "op": "checkpoint", "rows": rows, "cols": cols, "dtype": dtype}


def listed():
    return [
        # One sample answered: a launch, one exchange in a workgroup.
        _norm("norm_one_row", 1, 1024, "bf16", "e4m3"),
        # A long minibatch of wide rows, its normed rows kept in 8 bits: memory.
        _norm("norm_long", 16384, 8192, "bf16", "e4m3"),
        # A small fp32 minibatch of a width that no tile divides.
        _norm_back("norm_back_ragged", 333, 4100, "f32", "f32"),
        # The backward pass of the long minibatch, its stored sum an 8-bit checkpoint.
        _norm_back("norm_back_long", 16384, 8192, "bf16", "e4m3"),
        # One sample answered: the weights are read once, nothing else counts.
        _product("product_one_row", 1, 4096, 4096, "bf16", "silu", "bf16", "bf16", "none", True),
        # An fp32 minibatch of a square net.
        _product("product_f32", 256, 4096, 4096, "f32", "sigmoid", "f32", "f32", "f32", True),
        # Odd sizes in every direction: rows that start at odd addresses.
        _product("product_ragged", 333, 1365, 1083, "bf16", "relu", "bf16", "bf16", "bf16", False),
        # A bf16 minibatch, the input in 8 bits, the output and what the backward pass needs kept in 8 bits.
        _product("product_8bit", 512, 8192, 8192, "bf16", "gelu", "e4m3", "e4m3", "e4m3", False),
        # The fp32 minibatch's backward pass.
        _product_back("product_back_f32", 256, 4096, 4096, "f32", "sigmoid", "f32", "f32"),
        # The largest: a long bf16 minibatch's backward pass out of 8-bit checkpoints.
        _product_back("product_back_8bit", 4096, 8192, 8192, "bf16", "gelu", "e4m3", "e4m3"),
        # A small activation kept in 8 bits and taken back.
        _checkpoint("checkpoint_small", 32, 256, "bf16"),
        # A long one.
        _checkpoint("checkpoint_long", 16384, 8192, "bf16"),
    ]


def _size(rng, low, high):
    """A size between low and high, even over the logarithm; a third of them as they fall, the others whole vectors."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    step = rng.choice([1, 8, 64])
    return max(low, min(high, n if n < 2 * step else n // step * step))


def draw(rng):
    op = rng.choice(["norm", "norm_back", "product", "product", "product_back", "product_back", "checkpoint"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("norm", "norm_back", "checkpoint"):
        cols = _size(rng, 8, 16384)
        rows = _size(rng, 1, max(1, min(16384, ELEMENTS * (2 if dtype == "bf16" else 1) // 2 // cols)))
        if op == "norm":
            return _unnamed(_norm("", rows, cols, dtype, rng.choice([dtype, "e4m3"])))
        if op == "norm_back":
            return _unnamed(_norm_back("", rows, cols, dtype, rng.choice([dtype, "e4m3"])))
        return _unnamed(_checkpoint("", rows, cols, dtype))
    outputs, inputs = _size(rng, 16, 8192), _size(rng, 16, 8192)
    # fp32 products run at a sixteenth of the rate of bf16 ones
    most = FLOPS // (1 if dtype == "bf16" else 16) // (2 * outputs * inputs)
    rows = _size(rng, 1, max(1, min(8192, most)))
    act = rng.choice(["none", "sigmoid", "relu", "silu", "gelu"])
    x = rng.choice([dtype, "e4m3"])
    if op == "product":
        return _unnamed(_product("", rows, outputs, inputs, dtype, act, x, rng.choice([dtype, "e4m3"]),
                                 rng.choice(["none", dtype, "e4m3"]), rng.random() < 0.5))
    return _unnamed(_product_back("", rows, outputs, inputs, dtype, act, x, rng.choice([dtype, "e4m3"])))


def _unnamed(case):
    del case["name"]
    return case


def _bytes(kind, rows, cols):
    if kind == "e4m3":
        return rows * (cols + -(-cols // GROUP))
    return rows * cols * {"f32": 4, "bf16": 2, "none": 0}[kind]


def work(case):
    dt, rows = case["dtype"], case["rows"]
    if case["op"] == "norm":        # x, branch, gain in; sum, y, 1/rms out
        c = case["cols"]
        return {"bytes": 3 * _bytes(dt, rows, c) + _bytes(case["out"], rows, c) + 4 * c + 4 * rows, "flops": 5 * rows * c}
    if case["op"] == "norm_back":   # dy, sum, gradient of the sum, gain, 1/rms in; dx, dgain out
        c = case["cols"]
        return {"bytes": 3 * _bytes(dt, rows, c) + _bytes(case["stored"], rows, c) + 8 * c + 4 * rows, "flops": 9 * rows * c}
    if case["op"] == "checkpoint":  # saved, then loaded
        c = case["cols"]
        return {"bytes": 2 * _bytes(dt, rows, c) + 2 * _bytes("e4m3", rows, c), "flops": 3 * rows * c}
    o, i = case["outputs"], case["inputs"]
    if case["op"] == "product":
        moved = (_bytes(case["x"], rows, i) + _bytes(dt, o, i) + 4 * o + _bytes(case["y"], rows, o)
                 + _bytes(case["z"], rows, o) + (_bytes(dt, rows, o) if case["residual"] else 0))
        return {"bytes": moved, "flops": 2 * rows * o * i}
    moved = (_bytes(dt, rows, o) + (_bytes(case["z"], rows, o) if case["act"] != "none" else 0)
             + _bytes(case["x"], rows, i) + 2 * _bytes(dt, o, i) + _bytes(dt, rows, i) + 4 * o)
    return {"bytes": moved, "flops": 4 * rows * o * i}


# ---- 8 bits, from the definition -------------------------------------------------------------------------------------
def _exponents(v):
    """Per group of 32 columns the least e >= -117 with max|v| <= 448 * 2^e (v: rows x whole groups x 32)."""
    m, e = torch.frexp(v.abs().amax(-1))                    # m in [1/2, 1); 448 = 0.875 * 2^9
    return torch.where(m > 0.875, e - 8, e - 9).clamp_(min=LOWEST)


def _groups(v):
    rows, cols = v.shape
    return torch.nn.functional.pad(v, (0, -cols % GROUP)).view(rows, -1, GROUP)


def _pack(v):
    """(codes, scales) of a matrix: codes as float8 values of the matrix's shape, scales as powers of two."""
    rows, cols = v.shape
    g = _groups(v)
    e = _exponents(g)
    codes = torch.ldexp(g, -e.unsqueeze(-1)).to(torch.float8_e4m3fn).view(rows, -1)[:, :cols]
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _eight(codes, scales):
    return {"codes": codes, "scales": scales}


def _values(stored, wide=torch.float32):
    """The values of a matrix in its storage type or in 8 bits, in 32 or 64 bits."""
    if isinstance(stored, torch.Tensor):
        return stored.to(wide)
    codes, scales, cols = stored
    rows = codes.shape[0]
    v = codes.view(torch.float8_e4m3fn).to(wide).view(rows, -1, GROUP)
    v = v * scales.view(torch.float8_e8m0fnu).to(wide).unsqueeze(-1)
    return v.view(rows, -1)[:, :cols]


def _kept(v, kind):
    """A result as it is kept: rounded to the storage type, or in 8 bits."""
    return _eight(*_pack(v)) if kind == "e4m3" else v.to(TYPES[kind])


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _stored(v, kind):
    """An input as a user's program has it: a tensor, or 8-bit codes (rows padded to whole groups), scales, columns."""
    if kind != "e4m3":
        return v.to(TYPES[kind])
    g = _groups(v)
    e = _exponents(g)
    codes = torch.ldexp(g, -e.unsqueeze(-1)).to(torch.float8_e4m3fn).view(torch.uint8).view(v.shape[0], -1)
    return codes, (e + 127).to(torch.uint8), v.shape[1]


def _matrix(stored):
    """The same for the package's calls."""
    import paper_1801_04928_amd as lf
    return stored if isinstance(stored, torch.Tensor) else lf.E4M3Matrix.of(*stored)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(std)

    def features(rows, cols):
        # activations of a trained net: some features are many times larger than the rest
        return normal(rows, cols).mul_(torch.exp(normal(cols, std=0.7)))

    dt, rows, s = TYPES[case["dtype"]], case["rows"], {"case": case}
    op = case["op"]
    if op in ("norm", "norm_back"):
        c = case["cols"]
        s["gain"] = 1 + normal(c, std=0.1)
        if op == "norm":
            s["x"], s["branch"] = features(rows, c).to(dt), normal(rows, c, std=0.5).to(dt)
        else:
            total = features(rows, c)
            s["rstd"] = torch.rsqrt(total.square().mean(1) + EPS)
            s["sum"] = _stored(total, case["stored"])
            s["dy"], s["dsum"] = normal(rows, c, std=1e-2).to(dt), normal(rows, c, std=1e-2).to(dt)
    elif op == "checkpoint":
        s["x"] = features(rows, case["cols"]).to(dt)
    else:
        o, i = case["outputs"], case["inputs"]
        s["x"] = _stored(normal(rows, i), case["x"])
        s["w"] = normal(o, i, std=i ** -0.5).to(dt)
        if op == "product":
            s["b"] = normal(o, std=0.1)
            s["residual"] = normal(rows, o).to(dt) if case["residual"] else None
        else:
            s["z"] = _stored(normal(rows, o), case["z"])
            s["dy"] = normal(rows, o, std=1e-2).to(dt)
    if own:
        s["plan"] = _plan(case, s)
    return s


def _plan(case, s):
    """What a program that uses the package keeps: the operator with its outputs and workspace."""
    import paper_1801_04928_amd as lf
    dt, rows, op = case["dtype"], case["rows"], case["op"]
    s.update({name: _matrix(s[name]) for name in ("x", "sum", "z") if name in s})
    passes = "backward" if op.endswith("_back") else "forward"
    if op in ("norm", "norm_back"):
        p = lf.RmsNorm(rows, case["cols"], dt, out=case.get("out", dt), eps=EPS, passes=passes, device=DEVICE)
        p.gain.copy_(s["gain"])
    elif op == "checkpoint":
        p = lf.E4M3Matrix(rows, case["cols"], device=DEVICE)
        s["loaded"] = torch.empty_like(s["x"])
    else:
        p = lf.Linear(rows, case["outputs"], case["inputs"], dt, act=case["act"], y=case.get("y", dt), z=case["z"],
                      passes=passes, device=DEVICE)
        p.set_params(s["w"], s.get("b"))
    return p


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


def _act(z, act):
    if act == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if act == "relu":
        return torch.where(z < 0, 0, z)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * 0.5 ** 0.5)
    return z


def _act_slope(z, act):
    if act == "sigmoid":
        a = 1 / (1 + torch.exp(-z))
        return a * (1 - a)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        a = 1 / (1 + torch.exp(-z))
        return a * (1 + z * (1 - a))
    if act == "gelu":
        return 0.5 * torch.erfc(-z * 0.5 ** 0.5) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    return torch.ones_like(z)


def _run_plain(s, case):
    dt, op = TYPES[case["dtype"]], case["op"]
    if op == "norm":
        total = s["x"].float() + s["branch"].float()
        rstd = torch.rsqrt(total.square().mean(1) + EPS)
        return {"sum": total.to(dt), "rstd": rstd, "y": _kept(total * rstd.unsqueeze(1) * s["gain"], case["out"])}
    if op == "norm_back":
        rstd, dy = s["rstd"].unsqueeze(1), s["dy"].float()
        h, t = _values(s["sum"]) * rstd, dy * s["gain"]
        dx = s["dsum"].float() + rstd * (t - h * (t * h).mean(1, keepdim=True))
        return {"dx": dx.to(dt), "dgain": (dy * h).sum(0)}
    if op == "checkpoint":
        codes, scales = _pack(s["x"].float())
        rows, cols = s["x"].shape
        loaded = _groups(codes.float()) * scales.float().unsqueeze(-1)
        return {**_eight(codes, scales), "loaded": loaded.view(rows, -1)[:, :cols].to(dt)}
    x, w = _values(s["x"]), s["w"].float()
    if op == "product":
        z = x @ w.T + s["b"]
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out = {"y": _kept(y, case["y"])}
        if case["z"] != "none":
            out["z"] = _kept(z, case["z"])
        return out
    dz = s["dy"].float()
    if case["act"] != "none":
        dz = dz * _act_slope(_values(s["z"]), case["act"])
    return {"dx": (dz @ w).to(dt), "dw": (dz.T @ x).to(dt), "db": dz.sum(0)}


def _out(m):
    """A result of the package's calls: a tensor, or the codes and scales of a matrix in 8 bits."""
    if isinstance(m, torch.Tensor):
        return m
    return _eight(m.codes[:, :m.cols].view(torch.float8_e4m3fn), m.scales.view(torch.float8_e8m0fnu))


def _run_own(s, case):
    p, op = s["plan"], case["op"]
    if op == "norm":
        y = p.forward(s["x"], s["branch"])
        return {"sum": p.sum, "rstd": p.rstd, "y": _out(y)}
    if op == "norm_back":
        dx = p.backward(s["dy"], s["dsum"], stored=s["sum"], rstd=s["rstd"])
        return {"dx": dx, "dgain": p.dgain}
    if op == "checkpoint":
        p.save(s["x"])
        return {**_out(p), "loaded": p.load(out=s["loaded"])}
    if op == "product":
        y = p.forward(s["x"], s["residual"])
        out = {"y": _out(y)}
        if case["z"] != "none":
            out["z"] = _out(p.z)
        return out
    dx = p.backward(s["dy"], s["x"], z=s["z"])
    return {"dx": dx, "dw": p.dw, "db": p.db}


# ---- the same from the definitions, in 64 bits -----------------------------------------------------------------------
def _kept_exactly(v, kind):
    if kind != "e4m3":
        return v
    rows, cols = v.shape
    g = torch.nn.functional.pad(v, (0, -cols % GROUP)).reshape(rows, -1, GROUP)
    top = g.abs().amax(-1)
    e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448))       # then put right next to a power of two
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
    e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e).clamp(min=LOWEST)
    codes = (g / torch.exp2(e).unsqueeze(-1)).float().to(torch.float8_e4m3fn).double()
    return _eight(codes.reshape(rows, -1)[:, :cols], torch.exp2(e))


def exact(case, seed):
    s, op, wide = prepare(case, seed), case["op"], torch.float64
    if op == "norm":
        total = s["x"].to(wide) + s["branch"].to(wide)
        rstd = 1 / torch.sqrt((total * total).sum(1) / case["cols"] + EPS)
        return {"sum": total, "rstd": rstd, "y": _kept_exactly(total * rstd[:, None] * s["gain"].to(wide), case["out"])}
    if op == "norm_back":
        h = _values(s["sum"], wide) * s["rstd"].to(wide)[:, None]
        dy = s["dy"].to(wide)
        t = dy * s["gain"].to(wide)
        along = (t * h).sum(1, keepdim=True) / case["cols"]
        return {"dx": s["dsum"].to(wide) + s["rstd"].to(wide)[:, None] * (t - h * along), "dgain": (dy * h).sum(0)}
    if op == "checkpoint":
        kept = _kept_exactly(s["x"].to(wide), "e4m3")
        wide_scales = kept["scales"].repeat_interleave(GROUP, 1)[:, :case["cols"]]
        return {**kept, "loaded": kept["codes"] * wide_scales}
    x, w = _values(s["x"], wide), s["w"].to(wide)

    def sigmoid(v):
        return torch.where(v >= 0, 1 / (1 + torch.exp(-v.abs())), torch.exp(-v.abs()) / (1 + torch.exp(-v.abs())))

    if op == "product":
        z = torch.mm(x, w.t().contiguous()) + s["b"].to(wide)
        y = {"none": lambda: z, "sigmoid": lambda: sigmoid(z), "relu": lambda: z.clamp(min=0),
             "silu": lambda: z * sigmoid(z), "gelu": lambda: 0.5 * z * torch.erfc(-z / math.sqrt(2))}[case["act"]]()
        if s["residual"] is not None:
            y = y + s["residual"].to(wide)
        out = {"y": _kept_exactly(y, case["y"])}
        if case["z"] != "none":
            out["z"] = _kept_exactly(z, case["z"])
        return out
    z = _values(s["z"], wide)
    a = sigmoid(z)
    slope = {"none": lambda: torch.ones_like(z), "sigmoid": lambda: a * sigmoid(-z), "relu": lambda: (z > 0).to(wide),
             "silu": lambda: a + z * a * sigmoid(-z),
             "gelu": lambda: 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}
    dz = s["dy"].to(wide) * slope[case["act"]]()
    return {"dx": torch.mm(dz, w), "dw": torch.mm(dz.t().contiguous(), x), "db": dz.sum(0)}
