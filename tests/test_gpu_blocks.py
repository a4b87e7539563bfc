"""Matrices in 8 bits with blocks of 128 and their products, on the GPU against the 64-bit reference; the bounds are the reference's."""
import pytest
import torch

import paper_1801_04928_amd as P
from tests import student_reference as R
from tests.student_util import DEV, Blocks, Dense, MARK, TYPE, near, near_blocks, near_rounded, same, values

pytestmark = pytest.mark.gpu
ACTS = ["none", "sigmoid", "relu", "silu", "gelu"]


def spread(seed, rows, cols, dtype):
    """Values whose groups have scales of their own, from 2^-60 to 2^60."""
    v = values(seed, rows, cols)
    g = values(seed + 1, -(-rows // 64), -(-cols // 64)) * 20
    v = v * torch.exp2(g.round()).repeat_interleave(64, 0)[:rows].repeat_interleave(64, 1)[:, :cols]
    return v.to(TYPE[dtype]).double()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", [(1, 1), (1, 300), (300, 1), (3, 5), (127, 129), (128, 128), (129, 127), (200, 513), (260, 255), (5, 1024)])
def test_save_and_load(rows, cols, dtype):
    x = spread(rows, rows, cols, dtype)
    for tiles in (False, True):
        for both in ((1, 1), (1, 0), (0, 1)):
            mx = Dense(rows, cols, dtype, x, rows % 3, 5)
            out, out_t = Blocks(rows, cols, tiles, pad_groups=1), Blocks(cols, rows, tiles, pad_groups=2)
            assert P.lf_block_save(rows, cols, mx.m, out.m if both[0] else None, out_t.m if both[1] else None) == P.LF_OK
            torch.cuda.synchronize()
            pack = R.pack_tiles if tiles else R.pack
            for m, v, there in ((out, x, both[0]), (out_t, x.t().contiguous(), both[1])):
                if not there:
                    assert bool((m.codes == 0x7f).all()) and bool((m.scales == 255).all())
                    continue
                codes, e = m.raw()
                want, want_e = pack(v)
                same("codes", codes, want)
                same("scales", e, want_e)
                back = Dense(*v.shape, dtype, None, 3, 2)
                assert P.lf_block_load(*v.shape, m.m, back.m) == P.LF_OK
                same("values", back.get(), (R.held_tiles if tiles else R.held)(v).to(TYPE[dtype]).double())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite_and_the_largest(dtype):
    x = values(1, 130, 260, dtype=dtype)
    top = torch.finfo(TYPE[dtype]).max
    x[0, 0], x[1, 131], x[5, 259] = float("inf"), -float("inf"), float("nan")
    x[129, 200], x[3, 3], x[64] = top, -top, 0.0
    x[70, 128:256] = float("nan")
    x[71] *= 2.0 ** -120                                     # below the smallest scale's
    x = x.to(TYPE[dtype]).double()
    for tiles in (False, True):
        m, m_t = Blocks(130, 260, tiles), Blocks(260, 130, tiles)
        assert P.lf_block_save(130, 260, Dense(130, 260, dtype, x).m, m.m, m_t.m) == P.LF_OK
        torch.cuda.synchronize()
        for got, v in ((m, x), (m_t, x.t().contiguous())):
            codes, e = got.raw()
            want, want_e = (R.pack_tiles if tiles else R.pack)(v)
            same("scales", e, want_e)
            same("codes", codes, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tiles", [False, True])
def test_save_of_many_blocks(tiles, dtype):
    rows, cols = 2050, 4300
    x = spread(1, rows, cols, dtype)
    mx, out, out_t = Dense(rows, cols, dtype, x, 1, 3), Blocks(rows, cols, tiles, pad_groups=1), Blocks(cols, rows, tiles)
    assert P.lf_block_save(rows, cols, mx.m, out.m, out_t.m) == P.LF_OK
    torch.cuda.synchronize()
    for m, v in ((out, x), (out_t, x.t().contiguous())):
        codes, e = m.raw()
        want, want_e = (R.pack_tiles if tiles else R.pack)(v)
        same("codes", codes, want)
        same("scales", e, want_e)
        del codes, e, want, want_e


# (rows, outputs, inputs): few rows, in each number of 16 and past it; the tiles' ends in every direction; contractions that are split
SIZES = [(1, 1, 1), (1, 16, 128), (1, 333, 777), (2, 40, 7), (3, 129, 1300), (16, 50, 260), (17, 65, 300), (32, 31, 129), (33, 257, 90), (45, 130, 1083),
         (64, 20, 2000), (65, 129, 70), (130, 260, 190), (128, 128, 128), (257, 140, 64), (300, 257, 259), (70, 30, 9000), (200, 333, 2600),
         (9, 40, 5200), (16, 20, 9000), (31, 33, 1900), (31, 33, 2100), (60, 18, 1000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, outputs, inputs", SIZES)
def test_forward(rows, outputs, inputs, dtype):
    x, w = values(1, rows, inputs, dtype=dtype), values(2, outputs, inputs, dtype=dtype, std=inputs ** -0.5)
    bias, residual = values(3, outputs, std=0.3), values(4, rows, outputs, dtype=dtype)
    gb = bias.float().to(DEV)
    nbytes = P.lf_block_linear_workspace_bytes(rows, outputs, inputs)
    eight_x = R.held(x)
    for k, (kind, w_tiles, act, with_bias, with_residual, out) in enumerate([
            ("dense", True, "gelu", True, True, dtype), ("eight", True, "none", False, False, dtype), ("eight", False, "silu", True, False, "e4m3_128"),
            ("dense", True, "sigmoid", True, False, "e4m3_128"), ("dense", False, "relu", False, True, dtype)]):
        mx = Dense(rows, inputs, dtype, x, k % 3, 3) if kind == "dense" else Blocks(rows, inputs, values=x, pad_groups=1)
        mw, mr = Blocks(outputs, inputs, w_tiles, w, pad_groups=k % 2), Dense(rows, outputs, dtype, residual, 1, 2)
        y, z = (Blocks(rows, outputs, pad_groups=1) if out == "e4m3_128" else Dense(rows, outputs, dtype, None, i, 3) for i in (1, 2))
        x_t = Blocks(inputs, rows, pad_groups=1) if kind == "dense" else None
        scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
        assert P.lf_block_linear_forward(rows, outputs, inputs, mx.m, mw.m, gb.data_ptr() if with_bias else 0, ACTS.index(act),
                                         mr.m if with_residual else None, y.m, z.m, x_t.m if x_t else None, scratch.data_ptr(), nbytes) == P.LF_OK
        torch.cuda.synchronize()
        assert bool((scratch[nbytes:] == 255).all())
        exact = out != "e4m3_128" and dtype == "f32"
        (v, e_v), (want, e_y) = R.epilogue(*R.product(eight_x, (R.held_tiles if w_tiles else R.held)(w), exact), bias if with_bias else None, act,
                                           residual if with_residual else None)
        for name, m, wanted, bound in (("z", z, v, e_v), ("y", y, want, e_y)):
            if out == "e4m3_128":
                near_blocks(name, m, wanted, bound)
            else:
                m.get()
                near_rounded(name, m.t, wanted, bound)
        if x_t:
            codes, e = x_t.raw()
            want, want_e = R.pack(x.t().contiguous())
            same("x_t", codes, want)
            same("scales of x_t", e, want_e)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, outputs, inputs", SIZES)
def test_backward(rows, outputs, inputs, dtype):
    """dz of relu and of no activation is exact before it is kept in 8 bits, so both products' operands are known."""
    x, w = values(1, rows, inputs, dtype=dtype), values(2, outputs, inputs, dtype=dtype, std=outputs ** -0.5)
    dy, z = values(3, rows, outputs, dtype=dtype, std=0.01), values(4, rows, outputs, dtype=dtype)
    x_t, w_t = x.t().contiguous(), w.t().contiguous()
    nbytes = P.lf_block_linear_backward_workspace_bytes(rows, outputs, inputs)
    for k, (act, kept, w_tiles, dw_type, wanted) in enumerate([("relu", dtype, True, dtype, (1, 1, 1)), ("none", dtype, False, "f32", (1, 1, 0)),
                                                               ("relu", "e4m3_128", True, dtype, (1, 0, 1)), ("none", dtype, True, dtype, (0, 1, 1)),
                                                               ("relu", dtype, True, dtype, (0, 0, 1))]):
        mdy, mz = Dense(rows, outputs, dtype, dy, k % 3, 2), Blocks(rows, outputs, values=z) if kept == "e4m3_128" else Dense(rows, outputs, dtype, z, 1, 1)
        mx, mw = Blocks(inputs, rows, values=x_t, pad_groups=1), Blocks(inputs, outputs, w_tiles, w_t, pad_groups=k % 2)
        dx, dw, db = Dense(rows, inputs, dtype, None, 2, 3), Dense(outputs, inputs, dw_type, None, 1, 3), torch.full((outputs + 1,), MARK, device=DEV)
        scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
        assert P.lf_block_linear_backward(rows, outputs, inputs, mdy.m, mz.m if act != "none" else None, ACTS.index(act), mx.m if wanted[1] else None,
                                          mw.m if wanted[0] else None, dx.m if wanted[0] else None, dw.m if wanted[1] else None,
                                          db.data_ptr() if wanted[2] else 0, scratch.data_ptr(), nbytes) == P.LF_OK
        torch.cuda.synchronize()
        assert bool((scratch[nbytes:] == 255).all())
        dz = dy * R.slope(R.held(z) if kept == "e4m3_128" else z, act)
        if wanted[0]:
            dx.get()
            held = R.held_tiles(w_t) if w_tiles else R.held(w_t)
            near_rounded("dx", dx.t, *R.product(R.held(dz), held, dtype == "f32"))
        if wanted[1]:
            dw.get()
            near_rounded("dw", dw.t, *R.product(R.held(dz.t().contiguous()), R.held(x_t), dw_type == "f32"))
        assert float(db[outputs]) == MARK
        if wanted[2]:
            near("db", db[:outputs], dz.sum(0), (rows + 40) * R.U * dz.abs().sum(0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, outputs, inputs", [(64, 5003, 4100), (17, 8200, 2100), (5, 40, 40000), (2100, 4210, 1150), (2500, 2100, 1000), (3000, 3333, 130)])
def test_forward_of_large_products(rows, outputs, inputs, dtype):
    """Few rows whose products go by tiles, and tiles of every size with ends in every direction."""
    x, w = values(1, rows, inputs, dtype=dtype), values(2, outputs, inputs, dtype=dtype, std=inputs ** -0.5)
    bias = values(3, outputs, std=0.3)
    p = P.BlockLinear(rows, outputs, inputs, dtype, act="silu", z=dtype, passes="forward")
    p.set_params(w.to(TYPE[dtype]).to(DEV), bias.float().to(DEV))
    p.forward(x.to(TYPE[dtype]).to(DEV))
    (v, e_v), (want, e_y) = R.epilogue(*R.product(R.held(x), R.held_tiles(w), dtype == "f32"), bias, "silu", None)
    near_rounded("z", p.z, v, e_v)
    near_rounded("y", p.y, want, e_y)


@pytest.mark.parametrize("act", ["sigmoid", "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_of_smooth_activations(act, dtype):
    """dz is off by some u before it is kept: codes next to a border may be either, and so may scales.  So every value lies between what dz less
    its error and dz plus it are kept as, with the least or the largest scale that its group may have."""
    rows, outputs, inputs = 150, 140, 135
    x, w = values(1, rows, inputs, dtype=dtype), values(2, outputs, inputs, dtype=dtype, std=outputs ** -0.5)
    dy, z = values(3, rows, outputs, dtype=dtype, std=0.01), values(4, rows, outputs, dtype=dtype, std=2)
    p = P.BlockLinear(rows, outputs, inputs, dtype, act=act, dw="f32", passes="backward")
    p.set_params(w.to(TYPE[dtype]).to(DEV))
    x_t = P.E4M3Blocks(inputs, rows).save(x.t().contiguous().float().to(DEV))
    dx = p.backward(dy.to(TYPE[dtype]).to(DEV), x_t, z.to(TYPE[dtype]).to(DEV))
    dz = dy * R.slope(z, act)
    # the slope's functions are off by 8 u of the result and of arguments up to z^2, with factors up to z
    e_dz = dy.abs() * 32 * R.U * (1 + z.abs()).pow(3) + R.U * dz.abs()

    def between(v, e):
        low, high = [], []
        for scale in {R.pack((v.abs() - e).clamp(min=0))[1], R.pack(v.abs() + e)[1]}:
            s = torch.exp2(scale.double()).repeat_interleave(128, 1)[:, :v.shape[1]]
            for d, kept in ((-1, low), (1, high)):
                kept.append(R.nearest_codes(((v + d * e) / s).clamp(-448, 448)) * s)
        return R.held(v), torch.maximum(*high) - torch.minimum(*low)

    for name, got, a, e, other in (("dx", dx, dz, e_dz, R.held_tiles(w.t().contiguous())),
                                   ("dw", p.dw, dz.t().contiguous(), e_dz.t().contiguous(), R.held(x.t().contiguous()))):
        held, width = between(a, e)
        want, bound = R.product(held, other, got.dtype == torch.float32)
        near_rounded(name, got, want, bound + width @ other.abs().t())
    near("db", p.db, dz.sum(0), e_dz.sum(0) + (rows + 40) * R.U * dz.abs().sum(0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, outputs, inputs", [(5, 70, 300), (40, 70, 300), (300, 200, 300), (600, 5000, 257)])
def test_spoiled_values_stay_where_they_belong(rows, outputs, inputs, dtype):
    """A NaN in the last row and column reaches its row of the result and no other; what lies behind the operands' ends, NaN codes and
    scales among it, reaches nothing."""
    x, w = values(1, rows, inputs, dtype=dtype), values(2, outputs, inputs, dtype=dtype)
    x[rows - 1, inputs - 1] = float("nan")
    w[outputs - 1, inputs - 1] = float("nan")
    for w_tiles in (True, False):
        mx, mw, y = Blocks(rows, inputs, values=x, pad_groups=1), Blocks(outputs, inputs, w_tiles, w, pad_groups=1), Dense(rows, outputs, dtype)
        nbytes = P.lf_block_linear_workspace_bytes(rows, outputs, inputs)
        scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
        assert P.lf_block_linear_forward(rows, outputs, inputs, mx.m, mw.m, 0, 0, None, y.m, None, None, scratch.data_ptr(), nbytes) == P.LF_OK
        got = y.get().isnan()
        want = torch.zeros_like(got)
        want[rows - 1] = True
        want[:, outputs - 1] = True
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 40, 150])
def test_scale_bytes_that_others_write(rows, dtype):
    """Bytes of the whole range: the largest and smallest that stand for numbers, and 255 for NaN.  246 is the largest of which every code
    is a number: 448 * 2^127, of 254, is none of fp32's, and in a result in fp32 counts as infinite."""
    outputs, inputs = 130, 256
    x, w = values(1, rows, inputs, dtype="bf16"), values(2, outputs, inputs, dtype="bf16")
    for x_byte, w_byte in ((254, 1), (246, 9), (1, 246), (60, 200), (127, 127)):
        mx, mw, y = Blocks(rows, inputs, values=x), Blocks(outputs, inputs, True, w), Dense(rows, outputs, dtype)
        (cx, _), (cw, _) = mx.raw(), mw.raw()
        mx.scales[:rows, :2] = x_byte
        mw.scales[:2, :2] = w_byte
        nbytes = P.lf_block_linear_workspace_bytes(rows, outputs, inputs)
        scratch = torch.empty(nbytes + 256, dtype=torch.uint8, device=DEV)

        def run():
            assert P.lf_block_linear_forward(rows, outputs, inputs, mx.m, mw.m, 0, 0, None, y.m, None, None, scratch.data_ptr(), nbytes) == P.LF_OK
            return y.get()
        run()
        # of a byte below 10 the values may be rounded to bf16, and below the normal numbers to what is left of them: 2^-8 of each
        want, bound = R.product(cx * 2.0 ** (x_byte - 127), cw * 2.0 ** (w_byte - 127), dtype == "f32")
        coarse = 2.0 ** -4 if min(x_byte, w_byte) < 10 else 0.0
        size = (cx * 2.0 ** (x_byte - 127)).abs() @ (cw * 2.0 ** (w_byte - 127)).abs().t()
        if x_byte < 254 or dtype == "bf16":
            near_rounded("y", y.t, want, bound + coarse * size)
        else:
            assert not bool(torch.isfinite(y.t).any())
            continue
        mx.scales[rows - 1, 1] = 255
        nan = run().isnan()
        assert bool(nan[rows - 1].all()) and not bool(nan[:rows - 1].any())


def test_workspaces_are_scratch_and_streams_the_current_one():
    """The same call gives the same bits whatever lay in its workspace; two streams with objects of their own do not meet."""
    rows, o, i = 130, 260, 1500
    x = [values(s, rows, i, dtype="bf16").bfloat16().to(DEV) for s in (1, 2)]
    w = values(3, o, i, dtype="bf16").bfloat16().to(DEV)
    dy = values(4, rows, o, dtype="bf16").bfloat16().to(DEV)
    objects = [P.BlockLinear(rows, o, i, act="gelu", z="bf16") for _ in range(2)]
    for p in objects:
        p.set_params(w)
    want = []
    for p, v in zip(objects, x):
        p._workspace.fill_(255)
        y = p.forward(v).clone()
        p._workspace.fill_(0)
        p.backward(dy)
        want.append([t.clone() for t in (y, p.z, p.dx, p.dw, p.db)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in objects]
    for _ in range(3):
        for p, v, s in zip(objects, x, streams):
            with torch.cuda.stream(s):
                p.forward(v)
                p.backward(dy)
    torch.cuda.synchronize()
    for p, kept in zip(objects, want):
        assert all(torch.equal(a, b) for a, b in zip((p.y, p.z, p.dx, p.dw, p.db), kept))


def test_capture_and_replay():
    """Two captured graphs whose operators share a workspace, replayed in turn with the weights changing under them."""
    rows, sizes = 70, ((260, 130), (90, 260))
    nbytes = max(f(rows, o, i) for f in (P.lf_block_linear_workspace_bytes, P.lf_block_linear_backward_workspace_bytes) for o, i in sizes)
    scratch = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    made, graphs, inputs = [], [], []
    for k, (o, i) in enumerate(sizes):
        p = P.BlockLinear(rows, o, i, act="relu", z="bf16", workspace=scratch)
        p.set_params(values(k, o, i, dtype="bf16").bfloat16().to(DEV), values(k + 5, o).float().to(DEV))
        x, dy = torch.zeros(rows, i, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, o, dtype=torch.bfloat16, device=DEV)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            p.refresh()
            p.forward(x)
            p.backward(dy)
        made.append(p)
        graphs.append(graph)
        inputs.append((x, dy))
    for seed in range(3):
        for k, (p, graph, (x, dy)) in enumerate(zip(made, graphs, inputs)):
            x.copy_(values(seed, *x.shape))
            dy.copy_(values(seed + 3, *dy.shape))
            p.w.mul_(1.5)
            graph.replay()
        for p, (x, dy) in zip(made, inputs):
            e = P.BlockLinear(rows, p.outputs, p.inputs, act="relu", z="bf16")
            e.set_params(p.w, p.b)
            y, dx = e.forward(x), e.backward(dy)
            torch.cuda.synchronize()
            assert torch.equal(p.y, y) and torch.equal(p.dx, dx) and torch.equal(p.dw, e.dw) and torch.equal(p.db, e.db)


def test_fewer_rows_and_none():
    p = P.BlockLinear(300, 40, 60, act="silu", z="bf16")
    p.set_params(values(1, 40, 60, dtype="bf16").bfloat16().to(DEV))
    x, dy = values(2, 300, 60, dtype="bf16").bfloat16().to(DEV), values(3, 300, 40, dtype="bf16").bfloat16().to(DEV)
    for n in (131, 1, 300):
        small = P.BlockLinear(n, 40, 60, act="silu", z="bf16")
        small.set_params(p.w)
        assert torch.equal(p.forward(x[:n]), small.forward(x[:n])) and torch.equal(p.backward(dy[:n]), small.backward(dy[:n]))
        assert torch.equal(p.dw, small.dw) and torch.equal(p.db, small.db)
    assert p.forward(x[:0]).shape == (0, 40) and p.backward(dy[:0]).shape == (0, 60)
    assert bool((p.dw == 0).all()) and bool((p.db == 0).all())
