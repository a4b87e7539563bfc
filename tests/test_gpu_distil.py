"""The distillation loss and its gradient on the GPU against the 64-bit reference; the bounds are the reference's."""
import pytest
import torch

import paper_1801_04928_amd as P
from tests import student_reference as R
from tests.student_util import DEV, Dense, MARK, TYPE, near, near_rounded, values

pytestmark = pytest.mark.gpu

# (rows, classes, top): one class, less than a chunk, each kernel's widest row and the next, ends in every place
SIZES = [(3, 1, 1), (4, 5, 3), (2, 7, 7), (5, 8, 2), (6, 100, 10), (3, 512, 64), (3, 513, 65), (2, 2048, 5), (2, 2051, 128), (2, 4097, 9), (2, 8200, 200),
         (2, 16385, 33), (2, 32768, 64), (2, 32775, 3), (2, 65537, 64), (1, 131072, 7), (2, 131080, 1024), (700, 40, 4)]


def case(rows, classes, top, seed=0, std=3.0, dtype="f32", top_dtype="f32"):
    z = values(seed, rows, classes, dtype=dtype, std=std)
    order = torch.argsort(values(seed + 1, rows, classes), 1)[:, :top].to(torch.int32)
    t = (z.gather(1, order.long()) + values(seed + 2, rows, top)).to(TYPE[top_dtype]).double()
    weight = values(seed + 3, rows).abs()
    return z, t, order, weight


def run(z, t, classes, T, weight, dtype="f32", top_dtype="f32", grad=True, loss=True, off=0, in_place=False):
    rows, n, top = z.shape[0], z.shape[1], t.shape[1]
    mz, mt = Dense(rows, n, dtype, z, off, 3), Dense(rows, top, top_dtype, t, 1, 2)
    order = torch.full((rows, top + 3), 1 << 30, dtype=torch.int32, device=DEV)          # (what lies between the rows is no class)
    order[:, :top] = classes.to(DEV)
    d = None if not grad else mz if in_place else Dense(rows, n, dtype, None, 2, 5)
    out = torch.full((rows + 1,), MARK, device=DEV)
    gw = None if weight is None else weight.float().to(DEV)
    assert P.lf_distil(rows, n, top, mz.m, mt.m, order.data_ptr(), order.shape[1], T, 0 if gw is None else gw.data_ptr(), out.data_ptr() if loss else 0,
                       d.m if grad else None) == P.LF_OK
    torch.cuda.synchronize()
    assert float(out[rows]) == MARK
    if grad and not in_place:
        d.get()
    return out[:rows], d.t if grad else None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, classes, top", SIZES)
def test_loss_and_gradient(rows, classes, top, dtype):
    for k, (T, top_dtype, weighted) in enumerate([(1.0, "f32", True), (2.0, "bf16", False), (0.5, dtype, True)]):
        z, t, order, weight = case(rows, classes, top, seed=k, dtype=dtype, top_dtype=top_dtype)
        weight = weight.float().double() if weighted else torch.ones(rows, dtype=torch.float64)
        r = R.distil(z, t, order, T, weight)
        loss, d = run(z, t, order, T, weight if weighted else None, dtype, top_dtype, off=k)
        near("loss", loss, *r["loss"])
        near_rounded("dlogits", d, *r["dlogits"])
        alone, _ = run(z, t, order, T, weight if weighted else None, dtype, top_dtype, grad=False, off=k)
        assert torch.equal(alone, loss)
        there, d2 = run(z, t, order, T, weight if weighted else None, dtype, top_dtype, off=k, in_place=True, loss=k != 1)
        assert torch.equal(d2, d) and (torch.equal(there, loss) if k != 1 else bool((there == MARK).all()))


# every kernel for many rows, each with rows that end in its last chunks
MANY = [7, 300, 513, 1024, 1025, 2047, 2049, 4095, 4100, 6145, 8191, 8200, 12289, 16380, 16385, 24577, 32767, 32770, 40961, 49153, 57345, 65535, 65544]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes", MANY)
def test_many_rows(classes, dtype):
    """More rows than a workgroup each can be given at once.  (The reference runs on the GPU in 64 bits.)"""
    rows, top, T = 600, min(classes, 70), 2.0
    z = values(1, rows, classes, dtype=dtype, std=3.0) if classes < 3000 else None
    if z is None:
        g = torch.Generator(device=DEV)
        g.manual_seed(classes)
        z = torch.randn(rows, classes, generator=g, device=DEV).mul_(3).to(TYPE[dtype]).double()
    z = z.to(DEV)
    order = torch.stack([torch.randperm(classes, generator=torch.Generator().manual_seed(r))[:top] for r in range(rows)]).to(torch.int32).to(DEV)
    t = (z.gather(1, order.long()) + values(2, rows, top).to(DEV)).float().double()
    order[3] = order[3, 0]
    order[5] = -1
    weight = values(3, rows).abs().float().double().to(DEV)
    weight[7] = 0
    r = R.distil(z, t, order, T, weight)
    p = P.Distillation(rows, classes, top, dtype, temperature=T)
    loss = p.forward(z.to(TYPE[dtype]), t.float(), order, weight.float())
    for name, got, (want, bound) in (("loss", loss, r["loss"]), ("dlogits", p.dlogits, r["dlogits"])):
        off = (got.double() - want).abs()
        assert bool((off <= bound + R.HALF[got.dtype] * (want.abs() + bound) + 1e-40).all()), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("classes, top", [(50, 6), (3000, 70), (140000, 6)])
def test_rows_without_entries_weights_of_zero_and_repeated_classes(classes, top, dtype):
    z, t, order, weight = case(8, classes, top, dtype=dtype)
    weight = weight.float().double()
    order[0] = -1                                  # no entry
    order[1, 1:] = -7                              # one
    t[2] = -float("inf")                           # none above minus infinity
    t[3, 0] = -float("inf")
    weight[4] = 0.0
    z[4], t[4] = float("nan"), float("nan")        # ... is not looked at
    order[5] = order[5, 0]                         # one class for all
    order[6, 1::2] = order[6, 0]
    z[7, 3] = -float("inf")                        # a class the student never takes
    order[7] = torch.where(order[7] == 3, 4, order[7])
    r = R.distil(torch.where(z.isnan(), 0.0, z), torch.where(t.isnan(), 0.0, t), order, 2.0, weight)
    loss, d = run(z, t, order, 2.0, weight, dtype)
    for row in (0, 2, 4):
        assert float(loss[row]) == 0 and bool((d[row] == 0).all())
    near("loss", loss, *r["loss"])
    near_rounded("dlogits", d, *r["dlogits"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_have_no_answer(dtype):
    """A class past the last, NaN, infinities: the row is NaN, visibly, and no other."""
    z, t, order, _ = case(9, 200, 6, dtype=dtype)
    order[0, 2], order[1, 0] = 200, 2 ** 31 - 1
    z[2, 7], z[3, 199] = float("nan"), float("inf")
    t[4, 1], t[5, 2] = float("nan"), float("inf")
    z[6] = -float("inf")
    loss, d = run(z, t, order, 1.0, None, dtype)
    assert [bool(v) for v in loss.isnan()] == [True] * 7 + [False] * 2
    assert [bool(v) for v in d.isnan().any(1)] == [True] * 7 + [False] * 2 and bool(d[:3].isnan().all())
    z, t, order, _ = case(1, 200, 6, dtype=dtype)
    z[0, int(order[0, 2])] = -float("inf")         # the teacher takes what the student never does
    loss, d = run(z, t, order, 1.0, None, dtype)
    assert float(loss) == float("inf") and bool(torch.isfinite(d).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_classes(dtype):
    """Logits of the type's lowest value, of minus infinity and of the largest: those classes get nothing, and a row of equal ones is even."""
    low = torch.finfo(TYPE[dtype]).min
    for T in (2.0 ** -20, 0.5, 1.0, 2.0 ** 20):
        z, t, order, _ = case(4, 300, 5, std=2.0, dtype=dtype)
        z[0, 100:], z[1, 50:] = low, -float("inf")
        z[2] = low
        z[3] = -low
        order[0], order[1] = torch.arange(5), torch.arange(5, 10)
        loss, d = run(z, t, order, T, None, dtype)
        assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(d).all())
        if T >= 0.5:
            r = R.distil(z, t, order, T, torch.ones(4, dtype=torch.float64))
            if T == 2.0 ** 20:                     # (so flat that the lowest value's classes count: what is compared is what 64 bits say)
                z0 = slice(1, 4)
            else:
                z0 = slice(0, 4)
                assert bool((d[:2, 100:] == 0).all())
            near_rounded("dlogits", d[z0], r["dlogits"][0][z0], r["dlogits"][1][z0])


def test_gradient_against_differences_of_the_loss():
    """Central differences of step h of the reference's loss, off by h^2 of third derivatives (at most T^-1 weight): the gradient in fp32 lies
    within that and its bound."""
    z, t, order, weight = case(3, 20, 4)
    T, h = 2.0, 1e-3
    _, d = run(z, t, order, T, weight)
    r = R.distil(z, t, order, T, weight.float().double())
    for k in range(20):
        e = torch.zeros_like(z)
        e[:, k] = h
        slope = (R.distil(z + e, t, order, T, weight)["loss"][0] - R.distil(z - e, t, order, T, weight)["loss"][0]) / (2 * h)
        near("dlogits", d[:, k], slope, r["dlogits"][1][:, k] + h * h * weight + 1e-7 * weight)


def test_object_serves_fewer_rows_and_graphs():
    z, t, order, weight = case(30, 900, 12, dtype="bf16")
    gz, gt, go, gw = z.bfloat16().to(DEV), t.float().to(DEV), order.to(DEV), weight.float().to(DEV)
    p = P.Distillation(30, 900, 12, temperature=2.0)
    loss, d = p.forward(gz, gt, go, gw).clone(), p.dlogits.clone()
    assert torch.equal(p.forward(gz[:7], gt[:7], go[:7], gw[:7]), loss[:7]) and torch.equal(p.dlogits, d[:7]) and p.dlogits.shape == (7, 900)
    assert p.forward(gz[:0], gt[:0], go[:0]).shape == (0,)
    inside = P.Distillation(30, 900, 12, temperature=2.0, dlogits=gz)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        inside.forward(gz, gt, go, gw)
    for seed in range(3):
        gz.copy_(values(seed, 30, 900))
        p.forward(gz, gt, go, gw)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(inside.loss, p.loss) and torch.equal(gz, p.dlogits)
