"""Backward passes that go the ways that small sizes do not, against the 64-bit reference (computed on the GPU); the bounds are the reference's."""
import pytest
import torch

import paper_1801_04928_amd as P
from tests import student_reference as R
from tests.operators_reference import from_eight, to_eight
from tests.student_routes import BACKWARD, NORM_BACK
from tests.student_util import DEV, MARK, TYPE, Blocks, Dense, near, near_rounded, values
from tests.test_gpu_operators import Eight

pytestmark = pytest.mark.gpu
EPS = 1e-5


def on_cpu(pair):
    return [v.cpu() for v in pair]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, outputs, inputs", [sizes for sizes, _ in BACKWARD])
def test_products(rows, outputs, inputs, dtype):
    """dz of relu and of no activation is exact before it is kept in 8 bits, so both products' operands are known."""
    x, w = values(1, rows, inputs, dtype=dtype).to(DEV), values(2, outputs, inputs, dtype=dtype, std=outputs ** -0.5).to(DEV)
    dy, z = values(3, rows, outputs, dtype=dtype, std=0.01).to(DEV), values(4, rows, outputs, dtype=dtype).to(DEV)
    x_t, w_t = x.t().contiguous(), w.t().contiguous()
    wanted = {}
    with torch.device(DEV):                                    # (where the reference makes what it starts from)
        mx, mw = Blocks(inputs, rows, values=x_t, pad_groups=1), Blocks(inputs, outputs, True, w_t, pad_groups=1)
        held_x, held_w = R.held(x_t), R.held_tiles(w_t)
        for act in ("relu", "none"):
            dz = dy * R.slope(z, act)
            for name, a, b, types in (("dx", R.held(dz), held_w, (dtype,)),
                                      ("dw", R.held(dz.t().contiguous()), held_x, {dtype, "f32"} if act == "none" else (dtype,))):
                for t in types:
                    wanted[act, name, t] = on_cpu(R.product(a, b, t == "f32"))
            wanted[act, "db"] = on_cpu((dz.sum(0), (rows + 40) * R.U * dz.abs().sum(0)))
    mdy, mz = Dense(rows, outputs, dtype, dy, 1, 2), Dense(rows, outputs, dtype, z, 3, 1)
    nbytes = P.lf_block_linear_backward_workspace_bytes(rows, outputs, inputs)
    for act, dw_type, which in (("relu", dtype, "dx dw db"), ("none", "f32", "dx dw db"), ("relu", dtype, "dw db"), ("relu", dtype, "dx")):
        dx, dw, db = Dense(rows, inputs, dtype, None, 2, 3), Dense(outputs, inputs, dw_type, None, 1, 3), torch.full((outputs + 1,), MARK, device=DEV)
        scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
        assert P.lf_block_linear_backward(rows, outputs, inputs, mdy.m, mz.m if act != "none" else None, P.LF_ACT_RELU if act == "relu" else P.LF_ACT_NONE,
                                          mx.m if "dw" in which else None, mw.m if "dx" in which else None, dx.m if "dx" in which else None,
                                          dw.m if "dw" in which else None, db.data_ptr() if "db" in which else 0, scratch.data_ptr(), nbytes) == P.LF_OK
        torch.cuda.synchronize()
        assert bool((scratch[nbytes:] == 255).all()) and float(db[outputs]) == MARK
        if "dx" in which:
            dx.get()
            near_rounded("dx", dx.t, *wanted[act, "dx", dtype])
        if "dw" in which:
            dw.get()
            near_rounded("dw", dw.t, *wanted[act, "dw", dw_type])
        if "db" in which:
            near("db", db[:outputs], *wanted[act, "db"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dz_of_many_blocks_from_z_in_8_bits(dtype):
    """648 blocks of 128 x 128, which eight rows a thread take."""
    rows, outputs, inputs = 3000, 3333, 130
    dy, z = values(3, rows, outputs, dtype=dtype, std=0.01), values(4, rows, outputs, dtype=dtype)
    x = values(1, rows, inputs, dtype=dtype)
    mdy, mz, mx = Dense(rows, outputs, dtype, dy, 1, 2), Blocks(rows, outputs, values=z, pad_groups=1), Blocks(inputs, rows, values=x.t().contiguous())
    dw, db = Dense(outputs, inputs, dtype, None, 1, 3), torch.full((outputs + 1,), MARK, device=DEV)
    nbytes = P.lf_block_linear_backward_workspace_bytes(rows, outputs, inputs)
    scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
    assert P.lf_block_linear_backward(rows, outputs, inputs, mdy.m, mz.m, P.LF_ACT_RELU, mx.m, None, None, dw.m, db.data_ptr(), scratch.data_ptr(),
                                      nbytes) == P.LF_OK
    torch.cuda.synchronize()
    assert bool((scratch[nbytes:] == 255).all()) and float(db[outputs]) == MARK
    with torch.device(DEV):
        dz = dy.to(DEV) * R.slope(R.held(z.to(DEV)), "relu")
        want = on_cpu(R.product(R.held(dz.t().contiguous()), R.held(x.t().contiguous().to(DEV)), dtype == "f32"))
        want_db = on_cpu((dz.sum(0), (rows + 40) * R.U * dz.abs().sum(0)))
    dw.get()
    near_rounded("dw", dw.t, *want)
    near("db", db[:outputs], *want_db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kept", ["storage", "e4m3"])
@pytest.mark.parametrize("rows, cols", [s for sizes in NORM_BACK.values() for s in sizes])
def test_layer_norms(rows, cols, kept, dtype):
    s, dy, dsum = values(1, rows, cols, dtype=dtype, mean=1), values(2, rows, cols, dtype=dtype, std=0.1), values(5, rows, cols, dtype=dtype, std=0.1)
    if kept == "e4m3":                                         # (61 rows again and again: each is found value by value)
        codes, scales = (torch.from_numpy(v)[torch.arange(rows) % 61] for v in to_eight(s[:61].numpy()))
        ms, held = Eight(rows, cols, pad_groups=1), torch.from_numpy(from_eight(codes.numpy(), scales.numpy()))
        ms.codes[:rows, :cols], ms.scales[:rows, :ms.groups] = codes.to(DEV), scales.to(DEV)
    else:
        ms, held = Dense(rows, cols, dtype, s, 1, 5), s
    mean, rstd = held.mean(1).float(), (held - held.mean(1, keepdim=True)).square().mean(1).add(EPS).rsqrt().float()
    mdy, md, dx = Dense(rows, cols, dtype, dy, 1, 2), Dense(rows, cols, dtype, dsum, 2, 3), Dense(rows, cols, dtype, None, 3, 1)
    dgain, dshift = (torch.full((cols + 1,), MARK, device=DEV) for _ in range(2))
    gain = values(4, cols, std=0.3, mean=1.0)
    g, gmean, grstd = gain.float().to(DEV), mean.to(DEV), rstd.to(DEV)
    nbytes = P.lf_layer_norm_workspace_bytes(rows, cols)
    scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
    assert P.lf_layer_norm_backward(rows, cols, mdy.m, ms.m, g.data_ptr(), gmean.data_ptr(), grstd.data_ptr(), md.m, dx.m, dgain.data_ptr(),
                                    dshift.data_ptr(), scratch.data_ptr() if nbytes else 0, nbytes) == P.LF_OK
    torch.cuda.synchronize()
    r = R.norm_backward(dy, held, gain, mean.double(), rstd.double(), dsum)
    dx.get()
    assert bool((scratch[nbytes:] == 255).all()) and float(dgain[cols]) == MARK and float(dshift[cols]) == MARK
    near_rounded("dx", dx.t, *r["dx"])
    near("dgain", dgain[:cols], *r["dgain"])
    near("dshift", dshift[:cols], *r["dshift"])
