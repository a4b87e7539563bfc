"""Operators for training and serving student nets of residual blocks, as cases that can be prepared, run and timed: the layer
norm with the residual's addition, the matrix product of operands in 8 bits with a scale for each block of 128 with bias,
activation and residual in its epilogue, the backward passes of both, and the distillation loss from a teacher's top logits
with its gradient.

`run` computes an operator in its plain form (`own` false: elementary torch operations in 32 bits, rounded once at the
end) or through this package's entry points (`own` true).  `exact` computes the same from the definition in 64 bits.

8 bits: e4m3 codes with one power-of-two scale (e8m0) for 128 columns of a row (activations, gradients) or for 128 x 128
values (weights); rows of codes are padded to whole groups, rows of scales to whole fours.  What a product contracts over lies
along the rows of both operands, so a backward pass takes transposed matrices: of the weights the same codes, of activations
and gradients codes of their own, whose groups lie along the samples.

Shapes: rows x cols for norms, rows x inputs times (outputs x inputs)^T for products, rows x classes for the loss.  The
ranges: 1 to 16384 rows, 8 to 16384 columns, products of 16 to 8192 inputs and outputs, 8 to 64000 classes with 1 to 128 top
ones, with sizes that are no multiple of anything among them."""
import math

import torch

own = False

GROUP = 128
LOWEST = -117                       # the smallest scale: 2^-117 times the smallest code is a normal bf16 number
ELEMENTS = 16384 * 8192             # the largest norm
FLOPS = 2 * 4096 * 8192 * 8192      # the largest single product (a backward pass is two of them)
LOGITS = 4096 * 64000               # the largest loss
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DEVICE = "cuda:0"
EPS = 1e-5


def _norm(name, rows, cols, dtype, out):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "out": out}


def _norm_back(name, rows, cols, dtype):
    return {"name": name, "op": "norm_back", "rows": rows, "cols": cols, "dtype": dtype}


def _product(name, rows, outputs, inputs, dtype, act, residual, train):
    return {"name": name, "op": "product", "rows": rows, "outputs": outputs, "inputs": inputs, "dtype": dtype, "act": act,
            "residual": residual, "train": train}


def _product_back(name, rows, outputs, inputs, dtype, act):
    return {"name": name, "op": "product_back", "rows": rows, "outputs": outputs, "inputs": inputs, "dtype": dtype, "act": act}


def _distil(name, rows, classes, top, dtype, temperature, grad):
    return {"name": name, "op": "distil", "rows": rows, "classes": classes, "top": top, "dtype": dtype,
            "temperature": temperature, "grad": grad}


def listed():
    return [
        # One sample answered, its normed row the 8-bit operand of the product that follows: a launch.
        _norm("norm_one_row", 1, 1024, "bf16", "e4m3_128"),
        # A long minibatch of wide rows: memory.
        _norm("norm_long", 16384, 8192, "bf16", "bf16"),
        # A small fp32 minibatch of a width that no tile divides.
        _norm_back("norm_back_ragged", 333, 4100, "f32"),
        # The backward pass of the long minibatch.
        _norm_back("norm_back_long", 16384, 8192, "bf16"),
        # One sample answered: the weights are read once, nothing else counts.
        _product("product_one_row", 1, 4096, 4096, "bf16", "silu", True, False),
        # A few dozen samples answered together, odd sizes in every direction: rows that start at odd addresses.
        _product("product_ragged", 45, 1365, 1083, "f32", "sigmoid", False, False),
        # A long minibatch's forward pass in training: the value before the activation and the transposed input are kept.
        _product("product_train", 4096, 8192, 8192, "bf16", "gelu", False, True),
        # An ordinary minibatch's backward pass, of rows that no tile divides.
        _product_back("product_back", 500, 2048, 2048, "bf16", "relu"),
        # The largest: a long minibatch's backward pass.
        _product_back("product_back_long", 4096, 8192, 8192, "bf16", "gelu"),
        # The loss of a held-out handful of samples, no gradient: a launch.
        _distil("distil_loss", 32, 1000, 10, "f32", 1.0, False),
        # An odd number of classes: rows that start at odd addresses.
        _distil("distil_ragged", 777, 10007, 33, "bf16", 2.0, True),
        # A long minibatch and many classes: memory.
        _distil("distil_long", 4096, 64000, 64, "bf16", 2.0, True),
    ]


def _size(rng, low, high):
    """A size between low and high, even over the logarithm; a third of them as they fall, the others whole vectors."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    step = rng.choice([1, 8, 64])
    return max(low, min(high, n if n < 2 * step else n // step * step))


def draw(rng):
    op = rng.choice(["norm", "norm_back", "product", "product", "product_back", "product_back", "distil", "distil"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("norm", "norm_back"):
        cols = _size(rng, 8, 16384)
        rows = _size(rng, 1, max(1, min(16384, ELEMENTS * (2 if dtype == "bf16" else 1) // 2 // cols)))
        return _unnamed(_norm("", rows, cols, dtype, rng.choice([dtype, "e4m3_128"])) if op == "norm" else _norm_back("", rows, cols, dtype))
    if op == "distil":
        classes = _size(rng, 8, 64000)
        rows = _size(rng, 1, max(1, min(16384, LOGITS * (2 if dtype == "bf16" else 1) // 2 // classes)))
        return _unnamed(_distil("", rows, classes, _size(rng, 1, min(128, classes)), dtype, rng.choice([0.5, 1.0, 2.0, 4.0]),
                                rng.random() < 0.75))
    outputs, inputs = _size(rng, 16, 8192), _size(rng, 16, 8192)
    rows = _size(rng, 1, max(1, min(8192, FLOPS // (2 * outputs * inputs))))
    if op == "product":
        return _unnamed(_product("", rows, outputs, inputs, dtype, rng.choice(["none", "sigmoid", "relu", "silu", "gelu"]),
                                 rng.random() < 0.5, rng.random() < 0.5))
    # (fp32 results would show which values of dz lie next to a border between two codes, by chance in any arithmetic of 32
    # bits: fp32 cases take activations whose slopes are exact)
    return _unnamed(_product_back("", rows, outputs, inputs, dtype,
                                  rng.choice(["none", "relu"] if dtype == "f32" else ["none", "sigmoid", "relu", "silu", "gelu"])))


def _unnamed(case):
    del case["name"]
    return case


def _bytes(kind, rows, cols):
    if kind == "e4m3_128":
        return rows * (cols + -(-cols // GROUP))
    return rows * cols * {"f32": 4, "bf16": 2}[kind]


def work(case):
    dt, rows = case["dtype"], case["rows"]
    if case["op"] == "norm":        # x, branch, gain, shift in; sum, y, mean, 1/deviation out
        c = case["cols"]
        return {"bytes": 3 * _bytes(dt, rows, c) + _bytes(case["out"], rows, c) + 8 * c + 8 * rows, "flops": 8 * rows * c}
    if case["op"] == "norm_back":   # dy, sum, gradient of the sum, gain, mean, 1/deviation in; dx, dgain, dshift out
        c = case["cols"]
        return {"bytes": 4 * _bytes(dt, rows, c) + 12 * c + 8 * rows, "flops": 12 * rows * c}
    if case["op"] == "distil":      # logits, the teacher's top ones and their classes in; the loss and the gradient out
        c, top = case["classes"], case["top"]
        return {"bytes": (2 if case["grad"] else 1) * _bytes(dt, rows, c) + rows * (8 * top + 8), "flops": 5 * rows * c}
    o, i = case["outputs"], case["inputs"]
    weights = o * i + -(-o // GROUP) * -(-i // GROUP)
    if case["op"] == "product":     # x, w, bias and residual in; y, and for training z and x^T out
        moved = _bytes(dt, rows, i) + weights + 4 * o + _bytes(dt, rows, o) * (2 if case["residual"] else 1)
        if case["train"]:
            moved += _bytes(dt, rows, o) + _bytes("e4m3_128", i, rows)
        return {"bytes": moved, "flops": 2 * rows * o * i}
    # dy, z, x^T, w^T in; dx, dw, db out
    moved = (_bytes(dt, rows, o) * (1 if case["act"] == "none" else 2) + _bytes("e4m3_128", i, rows) + weights
             + _bytes(dt, rows, i) + _bytes(dt, o, i) + 4 * o)
    return {"bytes": moved, "flops": 4 * rows * o * i}


# ---- 8 bits, from the definition -------------------------------------------------------------------------------------
def _exponents(top):
    """The least e >= -117 with top <= 448 * 2^e."""
    m, e = torch.frexp(top)                                 # m in [1/2, 1); 448 = 0.875 * 2^9
    return torch.where(m > 0.875, e - 8, e - 9).clamp_(min=LOWEST)


def _groups(v):
    rows, cols = v.shape
    return torch.nn.functional.pad(v, (0, -cols % GROUP)).view(rows, -1, GROUP)


def _pack(v):
    """(codes as float8 values of the matrix's shape, exponents [rows][groups]) of a matrix, groups along its rows."""
    rows, cols = v.shape
    g = _groups(v)
    e = _exponents(g.abs().amax(-1))
    codes = torch.ldexp(g, -e.unsqueeze(-1)).to(torch.float8_e4m3fn).view(rows, -1)[:, :cols]
    return codes, e


def _pack_tiles(v):
    """The same with a scale for 128 x 128 values."""
    rows, cols = v.shape
    g = torch.nn.functional.pad(v, (0, -cols % GROUP, 0, -rows % GROUP)).view(-(-rows // GROUP), GROUP, -(-cols // GROUP), GROUP)
    e = _exponents(g.abs().amax((1, 3)))
    codes = torch.ldexp(g, -e[:, None, :, None]).to(torch.float8_e4m3fn).view(-(-rows // GROUP) * GROUP, -1)[:rows, :cols]
    return codes.contiguous(), e


def _unpack(codes, e, wide=torch.float32):
    """The values, in 32 or 64 bits."""
    rows, cols = codes.shape
    return (_groups(codes.to(wide)) * torch.exp2(e.to(wide)).unsqueeze(-1)).view(rows, -1)[:, :cols]


def _unpack_tiles(codes, e, wide=torch.float32):
    rows, cols = codes.shape
    scales = torch.exp2(e.to(wide)).repeat_interleave(GROUP, 0)[:rows].repeat_interleave(GROUP, 1)[:, :cols]
    return codes.to(wide) * scales


def _eight(codes, e):
    return {"codes": codes, "scales": (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)}


def _kept(v, kind):
    """A result as it is kept: rounded to the storage type, or in 8 bits."""
    return _eight(*_pack(v)) if kind == "e4m3_128" else v.to(TYPES[kind])


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _stored(codes, e):
    """A matrix in 8 bits as a user's program has it: codes with rows padded to whole groups, scale bytes to whole fours."""
    groups = -(-codes.shape[1] // GROUP)
    wide = torch.zeros(codes.shape[0], groups * GROUP, dtype=torch.uint8, device=DEVICE)
    wide[:, :codes.shape[1]] = codes.contiguous().view(torch.uint8)
    scales = torch.full((e.shape[0], -(-groups // 4) * 4), 127, dtype=torch.uint8, device=DEVICE)
    scales[:, :groups] = (e + 127).to(torch.uint8)
    return wide, scales


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEVICE).mul_(std)

    def features(rows, cols):
        # activations of a trained net: some features are many times larger than the rest, and have a mean of their own
        return normal(rows, cols).add_(normal(cols, std=0.3)).mul_(torch.exp(normal(cols, std=0.7)))

    dt, rows, op, s = TYPES[case["dtype"]], case["rows"], case["op"], {"case": case}
    if op in ("norm", "norm_back"):
        c = case["cols"]
        s["gain"], s["shift"] = 1 + normal(c, std=0.1), normal(c, std=0.1)
        if op == "norm":
            s["x"], s["branch"] = features(rows, c).to(dt), normal(rows, c, std=0.5).to(dt)
        else:
            total = features(rows, c)
            s["mean"] = total.mean(1)
            s["rstd"] = torch.rsqrt((total - s["mean"].unsqueeze(1)).square().mean(1) + EPS)
            s["sum"] = total.to(dt)
            s["dy"], s["dsum"] = normal(rows, c, std=1e-2).to(dt), normal(rows, c, std=1e-2).to(dt)
    elif op == "distil":
        c, top = case["classes"], case["top"]
        # the student's logits lie near the teacher's; the teacher's top ones come with their classes, in no order but theirs
        teacher = normal(rows, c, std=3.0)
        s["logits"] = (teacher + normal(rows, c)).to(dt)
        values, classes = torch.topk(teacher, top, dim=1)
        s["top_logits"], s["top_classes"] = values.to(dt), classes.to(torch.int32)
        # rows of padding count for nothing, the others for their share
        s["weight"] = (torch.rand(rows, generator=g, device=DEVICE) < 0.9).float() / rows
        s["weight"][0] = 1 / rows
    else:
        o, i = case["outputs"], case["inputs"]
        s["w"] = normal(o, i, std=i ** -0.5).to(dt)
        s["w8"] = _pack_tiles(s["w"].float())
        if op == "product":
            s["x"] = features(rows, i).to(dt)
            s["b"] = normal(o, std=0.1)
            s["residual"] = normal(rows, o).to(dt) if case["residual"] else None
        else:
            s["x_t"] = _pack(features(rows, i).to(dt).float().t().contiguous())
            s["z"] = normal(rows, o).to(dt)
            s["dy"] = normal(rows, o, std=1e-2).to(dt)
    if own:
        s["plan"] = _plan(case, s)
    return s


def _plan(case, s):
    """What a program that uses the package keeps: the operator with its outputs and workspace, the weights in 8 bits."""
    import paper_1801_04928_amd as lf
    dt, rows, op = case["dtype"], case["rows"], case["op"]
    if op in ("norm", "norm_back"):
        p = lf.LayerNorm(rows, case["cols"], dt, out=case.get("out", dt), eps=EPS, passes="forward" if op == "norm" else "backward",
                         device=DEVICE)
        p.gain.copy_(s["gain"])
        p.shift.copy_(s["shift"])
        return p
    if op == "distil":
        return lf.Distillation(rows, case["classes"], case["top"], dt, temperature=case["temperature"],
                               passes="both" if case["grad"] else "forward", device=DEVICE)
    passes = "backward" if op == "product_back" else "both" if case["train"] else "forward"
    p = lf.BlockLinear(rows, case["outputs"], case["inputs"], dt, act=case["act"], z=dt if passes == "both" else "none",
                       passes=passes, device=DEVICE)
    p.set_params(s["w"], s.get("b"))
    if op == "product_back":
        s["x_t_kept"] = lf.E4M3Blocks.of(*_stored(*s["x_t"]), rows)
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
        e = torch.exp(-z.abs())
        return e / (1 + e) ** 2
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
        mean = total.mean(1)
        off = total - mean.unsqueeze(1)
        rstd = torch.rsqrt(off.square().mean(1) + EPS)
        return {"sum": total.to(dt), "mean": mean, "rstd": rstd,
                "y": _kept(off * rstd.unsqueeze(1) * s["gain"] + s["shift"], case["out"])}
    if op == "norm_back":
        rstd, dy = s["rstd"].unsqueeze(1), s["dy"].float()
        h, t = (s["sum"].float() - s["mean"].unsqueeze(1)) * rstd, dy * s["gain"]
        dx = s["dsum"].float() + rstd * (t - t.mean(1, keepdim=True) - h * (t * h).mean(1, keepdim=True))
        return {"dx": dx.to(dt), "dgain": (dy * h).sum(0), "dshift": dy.sum(0)}
    if op == "distil":
        return _distil_plain(s, case)
    w = _unpack_tiles(*s["w8"])
    if op == "product":
        x = s["x"].float()
        z = _unpack(*_pack(x)) @ w.T + s["b"]
        y = _act(z, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out = {"y": y.to(dt)}
        if case["train"]:
            out["z"] = z.to(dt)
            out["x_t"] = _eight(*_pack(x.t().contiguous()))
        return out
    dz = s["dy"].float()
    if case["act"] != "none":
        dz = dz * _act_slope(s["z"].float(), case["act"])
    return {"dx": (_unpack(*_pack(dz)) @ w).to(dt),
            "dw": (_unpack(*_pack(dz.t().contiguous())) @ _unpack(*s["x_t"]).t()).to(dt), "db": dz.sum(0)}


def _distil_plain(s, case):
    """Of a row with weight g, temperature T, student z, teacher t over its top classes:  p = softmax(t / T),
    q = softmax(z / T) over all classes,  loss = g T^2 sum p (log p - log q),  dz = g T (q - p).  Weight 0: zeros."""
    T, classes = case["temperature"], s["top_classes"].long()
    z, t = s["logits"].float() / T, s["top_logits"].float() / T
    z = z - z.amax(1, keepdim=True)
    t = t - t.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    log_q = z.gather(1, classes) - torch.log(total)
    f = torch.exp(t)
    among = f.sum(1, keepdim=True)
    p, log_p = f / among, t - torch.log(among)
    g = s["weight"]
    out = {"loss": torch.where(g == 0, 0, g * T * T * (p * (log_p - log_q)).sum(1))}
    if case["grad"]:
        d = e / total
        d.scatter_add_(1, classes, -p)
        out["dlogits"] = torch.where(g.unsqueeze(1) == 0, 0, (g * T).unsqueeze(1) * d).to(s["logits"].dtype)
    return out


def _out(m):
    """A result of the package's calls: a tensor, or the codes and scales of a matrix in 8 bits."""
    if isinstance(m, torch.Tensor):
        return m
    groups = -(-m.cols // GROUP)
    return {"codes": m.codes[:, :m.cols].view(torch.float8_e4m3fn), "scales": m.scales[:, :groups].view(torch.float8_e8m0fnu)}


def _run_own(s, case):
    p, op = s["plan"], case["op"]
    if op == "norm":
        y = p.forward(s["x"], s["branch"])
        return {"sum": p.sum, "mean": p.mean, "rstd": p.rstd, "y": _out(y)}
    if op == "norm_back":
        dx = p.backward(s["dy"], s["dsum"], stored=s["sum"], mean=s["mean"], rstd=s["rstd"])
        return {"dx": dx, "dgain": p.dgain, "dshift": p.dshift}
    if op == "distil":
        loss = p.forward(s["logits"], s["top_logits"], s["top_classes"], s["weight"])
        return {"loss": loss, "dlogits": p.dlogits} if case["grad"] else {"loss": loss}
    if op == "product":
        y = p.forward(s["x"], s["residual"])
        return {"y": y, "z": p.z, "x_t": _out(p.x_t)} if case["train"] else {"y": y}
    dx = p.backward(s["dy"], s["x_t_kept"], z=s["z"])
    return {"dx": dx, "dw": p.dw, "db": p.db}


# ---- the same from the definitions, in 64 bits -----------------------------------------------------------------------
def _packed_exactly(v):
    """(codes' values, scales) in 64 bits."""
    rows, cols = v.shape
    g = torch.nn.functional.pad(v, (0, -cols % GROUP)).reshape(rows, -1, GROUP)
    top = g.abs().amax(-1)
    e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448))       # then put right next to a power of two
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
    e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e).clamp(min=LOWEST)
    codes = (g / torch.exp2(e).unsqueeze(-1)).float().to(torch.float8_e4m3fn).double()
    return codes.reshape(rows, -1)[:, :cols], torch.exp2(e)


def _eight_exactly(v):
    codes, scales = _packed_exactly(v)
    return {"codes": codes, "scales": scales}


def _held_exactly(v):
    """What a matrix in 8 bits holds of v."""
    codes, scales = _packed_exactly(v)
    return codes * scales.repeat_interleave(GROUP, 1)[:, :v.shape[1]]


def exact(case, seed):
    s, op, wide = prepare(case, seed), case["op"], torch.float64
    if op == "norm":
        total = s["x"].to(wide) + s["branch"].to(wide)
        mean = total.sum(1) / case["cols"]
        off = total - mean[:, None]
        rstd = 1 / torch.sqrt((off * off).sum(1) / case["cols"] + EPS)
        y = off * rstd[:, None] * s["gain"].to(wide) + s["shift"].to(wide)
        return {"sum": total, "mean": mean, "rstd": rstd, "y": _eight_exactly(y) if case["out"] == "e4m3_128" else y}
    if op == "norm_back":
        h = (s["sum"].to(wide) - s["mean"].to(wide)[:, None]) * s["rstd"].to(wide)[:, None]
        dy = s["dy"].to(wide)
        t = dy * s["gain"].to(wide)
        along, level = (t * h).sum(1, keepdim=True) / case["cols"], t.sum(1, keepdim=True) / case["cols"]
        return {"dx": s["dsum"].to(wide) + s["rstd"].to(wide)[:, None] * (t - level - h * along), "dgain": (dy * h).sum(0),
                "dshift": dy.sum(0)}
    if op == "distil":
        T, g, classes = case["temperature"], s["weight"].to(wide), s["top_classes"].long()
        log_q = torch.log_softmax(s["logits"].to(wide) / T, 1)
        log_p = torch.log_softmax(s["top_logits"].to(wide) / T, 1)
        p = torch.exp(log_p)
        out = {"loss": g * T * T * (p * (log_p - log_q.gather(1, classes))).sum(1)}
        if case["grad"]:
            d = torch.exp(log_q)
            d.scatter_add_(1, classes, -p)
            out["dlogits"] = d.mul_((g * T)[:, None])
        return out
    codes, e = s["w8"]
    w = codes.to(wide) * torch.exp2(e.to(wide)).repeat_interleave(GROUP, 0)[:codes.shape[0]].repeat_interleave(GROUP, 1)[:, :codes.shape[1]]

    def sigmoid(v):
        return torch.where(v >= 0, 1 / (1 + torch.exp(-v.abs())), torch.exp(-v.abs()) / (1 + torch.exp(-v.abs())))

    if op == "product":
        x = s["x"].to(wide)
        z = torch.mm(_held_exactly(x), w.t().contiguous()) + s["b"].to(wide)
        y = {"none": lambda: z, "sigmoid": lambda: sigmoid(z), "relu": lambda: z.clamp(min=0),
             "silu": lambda: z * sigmoid(z), "gelu": lambda: 0.5 * z * torch.erfc(-z / math.sqrt(2))}[case["act"]]()
        if s["residual"] is not None:
            y = y + s["residual"].to(wide)
        return {"y": y, "z": z, "x_t": _eight_exactly(x.t().contiguous())} if case["train"] else {"y": y}
    z = s["z"].to(wide)
    a = sigmoid(z)
    slope = {"none": lambda: torch.ones_like(z), "sigmoid": lambda: a * sigmoid(-z), "relu": lambda: (z > 0).to(wide),
             "silu": lambda: a + z * a * sigmoid(-z),
             "gelu": lambda: 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}
    dz = s["dy"].to(wide) * slope[case["act"]]()
    codes, e = s["x_t"]
    x_t = codes.to(wide) * torch.exp2(e.to(wide)).repeat_interleave(GROUP, 1)[:, :codes.shape[1]]
    return {"dx": torch.mm(_held_exactly(dz), w), "dw": torch.mm(_held_exactly(dz.t().contiguous()), x_t.t().contiguous()),
            "db": dz.sum(0)}
