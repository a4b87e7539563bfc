"""The layer norm on the GPU against the 64-bit reference; the bounds are the reference's."""
import pytest
import torch

import paper_1801_04928_amd as P
from tests import student_reference as R
from tests.student_util import DEV, Blocks, Dense, MARK, TYPE, near, near_blocks, near_rounded, values
from tests.operators_reference import from_eight, to_eight
from tests.test_gpu_operators import Eight

pytestmark = pytest.mark.gpu
EPS = 1e-5
F32_EPS = float(torch.tensor(EPS))

# one row to several a workgroup; a value, less than a chunk, ends in every place, each kernel's widest row and the next
SIZES = [(1, 1), (3, 5), (2, 7), (5, 8), (1, 1024), (9, 131), (7, 512), (6, 513), (5, 1025), (3, 4096), (4, 4097), (3, 8192), (2, 8200),
         (3, 16384), (2, 16385), (2, 20003), (37, 300), (130, 40)]


def vector(seed, n, mean=0.0):
    v = values(seed, n, std=0.3, mean=mean)
    return v, v.float().to(DEV)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", SIZES)
def test_forward(rows, cols, dtype):
    x, branch = values(1, rows, cols, dtype=dtype, std=2, mean=3), values(2, rows, cols, dtype=dtype)
    (gain, g), (shift, b) = vector(3, cols, 1.0), vector(4, cols)
    for k, (out, with_branch, plain) in enumerate([(dtype, True, False), ("e4m3_128", True, False), ("e4m3", False, True), (dtype, False, True)]):
        off, pad = k % 3, (5, 8, 3)[k % 3]
        mx, mb = Dense(rows, cols, dtype, x, off, pad), Dense(rows, cols, dtype, branch, 1, 3)
        total = Dense(rows, cols, dtype, None, 3, 2) if with_branch else None
        y = {"e4m3_128": lambda: Blocks(rows, cols, pad_groups=1), "e4m3": lambda: Eight(rows, cols, pad_groups=1)}.get(out, lambda: Dense(rows, cols, dtype, None, 2, 7))()
        mean, rstd = torch.full((rows + 1,), MARK, device=DEV), torch.full((rows + 1,), MARK, device=DEV)
        assert P.lf_layer_norm_forward(rows, cols, mx.m, mb.m if with_branch else None, 0 if plain else g.data_ptr(), 0 if plain else b.data_ptr(), EPS,
                                       total.m if total else None, y.m, mean.data_ptr(), rstd.data_ptr()) == P.LF_OK
        torch.cuda.synchronize()
        one, zero = torch.ones(cols, dtype=torch.float64), torch.zeros(cols, dtype=torch.float64)
        r = R.norm_forward(x, branch if with_branch else None, one if plain else gain, zero if plain else shift, F32_EPS)
        assert float(mean[rows]) == MARK and float(rstd[rows]) == MARK
        near("mean", mean[:rows], *r["mean"])
        near("rstd", rstd[:rows], *r["rstd"])
        if total:
            total.get()
            near_rounded("sum", total.t, *r["sum"])
        if out == "e4m3_128":
            near_blocks("y", y, *r["y"])
        elif out == "e4m3":
            want, bound = r["y"]
            codes, scales = y.raw()
            scale = torch.exp2(torch.from_numpy(scales).double() - 127).repeat_interleave(32, 1)[:, :cols]
            near("y", torch.from_numpy(y.get()), want, bound + torch.maximum(2.0 ** -4 * (want.abs() + bound), 2.0 ** -10 * scale))
        else:
            y.get()
            near_rounded("y", y.t, *r["y"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_mean_far_from_zero_keeps_the_digits(dtype):
    """A row of 4096 + {0, 32}: the difference of two sums of squares would keep none of the variance's."""
    x = 4096 + 32 * (torch.arange(4 * 300).view(4, 300) % 3 == 0).double()
    n = P.LayerNorm(4, 300, dtype, eps=0.0)
    y = n.forward(x.to(TYPE[dtype]).to(DEV))
    r = R.norm_forward(x, None, torch.ones(300, dtype=torch.float64), torch.zeros(300, dtype=torch.float64), 0.0)
    near("rstd", n.rstd, *r["rstd"])
    near_rounded("y", y, *r["y"])
    assert float((n.rstd.double().cpu() / r["rstd"][0] - 1).abs().max()) < 1e-2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_values_and_spoiled_rows(dtype):
    """A row without variance comes out as the shift; infinities and NaN spoil their own row alone."""
    x = values(1, 6, 140, dtype=dtype)
    x[1] = 2.5
    x[3, 139], x[4, 0] = float("inf"), float("nan")
    n = P.LayerNorm(6, 140, dtype)
    n.shift.fill_(0.75)
    y = n.forward(x.to(TYPE[dtype]).to(DEV)).double().cpu()
    assert bool((y[1] == 0.75).all())
    assert [bool(v) for v in y.isnan().all(1)] == [False, False, False, True, True, False] and bool(torch.isfinite(y[[0, 1, 2, 5]]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", SIZES)
def test_backward(rows, cols, dtype):
    s, dy = values(1, rows, cols, dtype=dtype, std=2, mean=1), values(2, rows, cols, dtype=dtype, std=0.1)
    dsum, (gain, g) = values(3, rows, cols, dtype=dtype, std=0.1), vector(4, cols, 1.0)
    for k, (kept, more, plain, wanted) in enumerate([(dtype, True, False, (1, 1)), ("e4m3", False, True, (1, 1)), (dtype, False, False, (1, 0)),
                                                     (dtype, True, True, (0, 1)), (dtype, True, False, (0, 0))]):
        off = k % 3
        ms = Eight(rows, cols, s.numpy(), pad_groups=1) if kept == "e4m3" else Dense(rows, cols, dtype, s, off, 5)
        held = torch.from_numpy(from_eight(*to_eight(s.numpy()))) if kept == "e4m3" else s
        mean = held.mean(1).float()
        rstd = (held - mean.double()[:, None]).square().mean(1).add(EPS).rsqrt().float()
        mdy, md, dx = Dense(rows, cols, dtype, dy, 1, 2), Dense(rows, cols, dtype, dsum, 2, 3), Dense(rows, cols, dtype, None, 3, 1)
        dgain, dshift = (torch.full((cols + 1,), MARK, device=DEV) for _ in range(2))
        nbytes = P.lf_layer_norm_workspace_bytes(rows, cols) if any(wanted) else 0
        scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
        gmean, grstd = mean.to(DEV), rstd.to(DEV)
        assert P.lf_layer_norm_backward(rows, cols, mdy.m, ms.m, 0 if plain else g.data_ptr(), gmean.data_ptr(), grstd.data_ptr(), md.m if more else None,
                                        dx.m, dgain.data_ptr() if wanted[0] else 0, dshift.data_ptr() if wanted[1] else 0,
                                        scratch.data_ptr() if nbytes else 0, nbytes) == P.LF_OK
        torch.cuda.synchronize()
        r = R.norm_backward(dy, held, torch.ones(cols, dtype=torch.float64) if plain else gain, mean.double(), rstd.double(), dsum if more else None)
        dx.get()
        assert bool((scratch[nbytes:] == 255).all())
        near_rounded("dx", dx.t, *r["dx"])
        for name, got, want in (("dgain", dgain, wanted[0]), ("dshift", dshift, wanted[1])):
            assert float(got[cols]) == MARK
            if want:
                near(name, got[:cols], *r[name])
            else:
                assert bool((got == MARK).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", [(1300, 200), (700, 2500), (600, 5000), (530, 9001), (1100, 17000)])
def test_backward_of_many_rows(rows, cols, dtype):
    """Workgroups that walk several rows, and partial sums in every order."""
    s, dy = values(1, rows, cols, dtype=dtype, mean=1), values(2, rows, cols, dtype=dtype, std=0.1)
    mean, rstd = s.mean(1).float(), (s - s.mean(1, keepdim=True)).square().mean(1).add(EPS).rsqrt().float()
    n = P.LayerNorm(rows, cols, dtype, passes="backward")
    dx = n.backward(dy.to(TYPE[dtype]).to(DEV), stored=s.to(TYPE[dtype]).to(DEV), mean=mean.to(DEV), rstd=rstd.to(DEV))
    r = R.norm_backward(dy, s, torch.ones(cols, dtype=torch.float64), mean.double(), rstd.double(), None)
    near_rounded("dx", dx, *r["dx"])
    near("dgain", n.dgain, *r["dgain"])
    near("dshift", n.dshift, *r["dshift"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", [(513, 5), (520, 700), (900, 70), (600, 9001)])
def test_backward_of_many_rows_in_8_bits(rows, cols, dtype):
    s, dy = values(1, rows, cols, dtype=dtype, mean=1), values(2, rows, cols, dtype=dtype, std=0.1)
    ms, mdy, dx = Eight(rows, cols, s.numpy(), pad_groups=1), Dense(rows, cols, dtype, dy, 1, 2), Dense(rows, cols, dtype, None, 3, 1)
    held = torch.from_numpy(from_eight(*to_eight(s.numpy())))
    mean, rstd = held.mean(1).float(), (held - held.mean(1, keepdim=True)).square().mean(1).add(EPS).rsqrt().float()
    dgain, dshift = (torch.full((cols + 1,), MARK, device=DEV) for _ in range(2))
    gain, g = vector(4, cols, 1.0)
    nbytes = P.lf_layer_norm_workspace_bytes(rows, cols)
    scratch = torch.full((nbytes + 256,), 255, dtype=torch.uint8, device=DEV)
    gmean, grstd = mean.to(DEV), rstd.to(DEV)
    assert P.lf_layer_norm_backward(rows, cols, mdy.m, ms.m, g.data_ptr(), gmean.data_ptr(), grstd.data_ptr(), None, dx.m, dgain.data_ptr(),
                                    dshift.data_ptr(), scratch.data_ptr(), nbytes) == P.LF_OK
    torch.cuda.synchronize()
    r = R.norm_backward(dy, held, gain, mean.double(), rstd.double(), None)
    dx.get()
    assert bool((scratch[nbytes:] == 255).all()) and float(dgain[cols]) == MARK and float(dshift[cols]) == MARK
    near_rounded("dx", dx.t, *r["dx"])
    near("dgain", dgain[:cols], *r["dgain"])
    near("dshift", dshift[:cols], *r["dshift"])


def test_outputs_in_the_inputs_place_and_fewer_rows():
    """sum may be x or branch, dx may be dsum; an object serves fewer rows than it was made for, and none."""
    x, branch = (values(i, 5, 70, dtype="bf16").bfloat16().to(DEV) for i in (1, 2))
    want = P.LayerNorm(5, 70)
    want.forward(x, branch)
    for place in (x, branch):
        mine = place.clone()
        n = P.LayerNorm(5, 70, sum=mine)
        y = n.forward(*((mine, branch) if place is x else (x, mine)))
        assert n.sum is mine and torch.equal(mine, want.sum) and torch.equal(y, want.y)
    dy, ds = (values(i, 5, 70, dtype="bf16").bfloat16().to(DEV) for i in (3, 4))
    dx = want.backward(dy, ds)
    n = P.LayerNorm(9, 70, dx=torch.cat([ds, ds])[:9])
    n.forward(x, branch)
    assert torch.equal(n.backward(dy, n._dx[:5]), dx) and torch.equal(n.dgain, want.dgain) and torch.equal(n.dshift, want.dshift)
    assert n.forward(x[:0]).shape == (0, 70) and n.backward(dy[:0]).shape == (0, 70)
    assert bool((n.dgain == 0).all()) and bool((n.dshift == 0).all())


def test_capture_and_replay():
    """A captured forward and backward pass, replayed with other inputs among the program's own work."""
    rows, cols = 65, 1030
    n = P.LayerNorm(rows, cols, "bf16", out="e4m3_128")
    x, dy = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV), torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    x.zero_()
    dy.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        n.forward(x)
        n.backward(dy)
    eager = P.LayerNorm(rows, cols, "bf16", out="e4m3_128")
    for seed in range(3):
        x.copy_(values(seed, rows, cols))
        dy.copy_(values(seed + 10, rows, cols))
        graph.replay()
        y = eager.forward(x)
        dx = eager.backward(dy)
        torch.cuda.synchronize()
        assert torch.equal(n.y.codes, y.codes) and torch.equal(n.y.scales[:, :9], y.scales[:, :9]) and torch.equal(n.dx, dx)
        assert torch.equal(n.dgain, eager.dgain) and torch.equal(n.dshift, eager.dshift)
