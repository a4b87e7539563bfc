"""Host-side checks of the student nets' operators (no GPU): arguments are refused before anything is enqueued, workspaces that serve
some rows serve fewer, and what the objects hand to the C calls."""
import pytest
import torch

import paper_1801_04928_amd as P
from tests.test_operators_objects import GPU, OnGpu, calls, given, on_gpu, tensor  # noqa: F401  (calls: a fixture)

FAKE = 1 << 20          # a "device pointer" that is only checked for alignment
F, B, E, R, T = P.LF_MATRIX_F32, P.LF_MATRIX_BF16, P.LF_MATRIX_E4M3, P.LF_MATRIX_E4M3_128, P.LF_MATRIX_E4M3_TILES


def mat(kind, ld, data=FAKE, scales=FAKE, scale_ld=None):
    if scale_ld is None:
        scale_ld = -(-ld // 32) if kind == E else -(-(-(-ld // 128)) // 4) * 4
    return P.lf_matrix(data, ld, scales if kind >= E else None, scale_ld, kind)


def norm(rows=4, cols=40, x=mat(B, 40), branch=None, gain=FAKE, shift=FAKE, eps=1e-5, total=mat(B, 40), y=mat(R, 128), mean=FAKE, rstd=FAKE):
    return P.lf_layer_norm_forward(rows, cols, x, branch, gain, shift, eps, total, y, mean, rstd)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(x=mat(R, 128)),
    dict(branch=mat(F, 40)), dict(branch=mat(B, 39)), dict(gain=FAKE + 2), dict(shift=FAKE + 1), dict(total=mat(R, 128)),
    dict(total=mat(F, 40)), dict(y=None), dict(y=mat(F, 40)), dict(y=mat(R, 64)), dict(y=mat(T, 128)), dict(y=mat(R, 192)),
    dict(y=mat(R, 128, scales=FAKE + 2)), dict(y=mat(R, 128, scale_ld=1)), dict(y=mat(R, 128, scale_ld=6)), dict(y=mat(R, 128, data=FAKE + 8)),
    dict(mean=FAKE + 1), dict(rstd=FAKE + 2)])
def test_layer_norm_forward_refusals(change):
    assert norm(**change) == P.LF_EINVAL
    assert "lf_layer_norm_forward" in P.lf_operator_error()


def norm_back(rows=2000, cols=40, dy=mat(B, 40), total=mat(B, 40), gain=FAKE, mean=FAKE, rstd=FAKE, dsum=None, dx=mat(B, 40), dgain=FAKE,
              dshift=FAKE, workspace=FAKE, nbytes=1 << 20):
    return P.lf_layer_norm_backward(rows, cols, dy, total, gain, mean, rstd, dsum, dx, dgain, dshift, workspace, nbytes)


@pytest.mark.parametrize("change", [
    dict(dy=None), dict(dy=mat(R, 128)), dict(total=None), dict(total=mat(F, 40)), dict(total=mat(R, 128)), dict(gain=FAKE + 2), dict(mean=0),
    dict(rstd=0), dict(mean=FAKE + 2), dict(dsum=mat(F, 40)), dict(dx=None), dict(dx=mat(F, 40)), dict(dgain=FAKE + 1), dict(dshift=FAKE + 1),
    dict(workspace=0), dict(workspace=FAKE + 16), dict(nbytes=0), dict(dgain=0, nbytes=0), dict(dshift=0, nbytes=0)])
def test_layer_norm_backward_refusals(change):
    assert norm_back(**change) == P.LF_EINVAL
    assert "lf_layer_norm_backward" in P.lf_operator_error()


def save(rows=4, cols=200, x=mat(B, 200), out=mat(R, 256), out_t=mat(R, 128)):
    return P.lf_block_save(rows, cols, x, out, out_t)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(x=None), dict(x=mat(E, 224)), dict(x=mat(R, 256)), dict(x=mat(B, 199)), dict(out=None, out_t=None),
    dict(out=mat(E, 224)), dict(out=mat(R, 128)), dict(out=mat(T, 256)), dict(out_t=mat(T, 128)), dict(out_t=mat(B, 4)), dict(rows=130),
    dict(out=mat(R, 256, scales=0)), dict(out=mat(R, 288)), dict(out=mat(T, 256), out_t=mat(R, 128))])
def test_block_save_refusals(change):
    assert save(**change) == P.LF_EINVAL
    assert "lf_block_save" in P.lf_operator_error()


def test_block_load_refusals():
    assert P.lf_block_load(4, 200, mat(E, 224), mat(B, 200)) == P.LF_EINVAL
    assert P.lf_block_load(4, 200, mat(R, 256), mat(R, 256)) == P.LF_EINVAL
    assert P.lf_block_load(4, 200, mat(T, 256), mat(B, 199)) == P.LF_EINVAL
    assert P.lf_block_load(4, 200, None, mat(B, 200)) == P.LF_EINVAL


def linear(rows=40, outputs=48, inputs=200, x=mat(B, 200), w=mat(T, 256), bias=FAKE, act=P.LF_ACT_GELU, residual=None, y=mat(B, 48),
           z=mat(B, 48), x_t=mat(R, 128), workspace=FAKE, nbytes=1 << 30):
    return P.lf_block_linear_forward(rows, outputs, inputs, x, w, bias, act, residual, y, z, x_t, workspace, nbytes)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(outputs=0), dict(inputs=0), dict(x=None), dict(x=mat(E, 224)), dict(x=mat(T, 256)), dict(w=None), dict(w=mat(B, 200)),
    dict(w=mat(E, 224)), dict(w=mat(T, 128)), dict(bias=FAKE + 2), dict(act=5), dict(act=-1), dict(residual=mat(F, 48)), dict(residual=mat(R, 128)),
    dict(y=None), dict(y=mat(F, 48)), dict(y=mat(T, 128)), dict(z=mat(F, 48)), dict(z=mat(E, 64)), dict(x_t=mat(T, 128)), dict(x_t=mat(B, 40)),
    dict(x=mat(R, 256)), dict(x=mat(R, 256), x_t=None, y=mat(F, 48)), dict(x=mat(R, 256), x_t=None, residual=mat(F, 48)),
    dict(workspace=0), dict(nbytes=64), dict(workspace=FAKE + 128)])
def test_block_linear_forward_refusals(change):
    assert linear(**change) == P.LF_EINVAL
    assert "lf_block_linear_forward" in P.lf_operator_error()


def linear_back(rows=40, outputs=48, inputs=200, dy=mat(B, 48), z=mat(B, 48), act=P.LF_ACT_SILU, x_t=mat(R, 128), w_t=mat(T, 128),
                dx=mat(B, 200), dw=mat(F, 200), db=FAKE, workspace=FAKE, nbytes=1 << 30):
    return P.lf_block_linear_backward(rows, outputs, inputs, dy, z, act, x_t, w_t, dx, dw, db, workspace, nbytes)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(outputs=0), dict(inputs=0), dict(dy=None), dict(dy=mat(R, 128)), dict(z=None), dict(z=mat(F, 48)), dict(z=mat(E, 64)),
    dict(act=9), dict(x_t=None), dict(x_t=mat(B, 40)), dict(x_t=mat(T, 128)), dict(w_t=None), dict(w_t=mat(B, 48)), dict(dx=mat(F, 200)),
    dict(dw=mat(R, 256)), dict(dw=mat(B, 199)), dict(db=FAKE + 2), dict(workspace=0), dict(nbytes=64), dict(rows=130)])
def test_block_linear_backward_refusals(change):
    assert linear_back(**change) == P.LF_EINVAL
    assert "lf_block_linear_backward" in P.lf_operator_error()


def distil(rows=4, classes=40, top=5, logits=mat(B, 40), top_logits=mat(F, 5), top_classes=FAKE, ld=5, temperature=2.0, weight=FAKE,
           loss=FAKE, dlogits=mat(B, 40)):
    return P.lf_distil(rows, classes, top, logits, top_logits, top_classes, ld, temperature, weight, loss, dlogits)


@pytest.mark.parametrize("change, status", [
    (c, P.LF_EINVAL) for c in (
        dict(rows=-1), dict(classes=0), dict(top=0), dict(logits=None), dict(logits=mat(R, 128)), dict(logits=mat(B, 39)), dict(top_logits=None),
        dict(top_logits=mat(F, 4)), dict(top_classes=0), dict(top_classes=FAKE + 2), dict(ld=4), dict(temperature=0.0), dict(temperature=-1.0),
        dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=2.0 ** -21), dict(temperature=2.0 ** 21),
        dict(weight=FAKE + 2), dict(loss=FAKE + 1), dict(dlogits=mat(F, 40)), dict(loss=0, dlogits=None))
] + [(dict(top=1025, top_logits=mat(F, 1025), ld=1025), P.LF_EUNSUPPORTED), (dict(ld=1 << 22), P.LF_EUNSUPPORTED)])
def test_distil_refusals(change, status):
    assert distil(**change) == status
    assert "lf_distil" in P.lf_operator_error()


def test_workspaces_serve_fewer_rows():
    for outputs, inputs in ((48, 8192), (8192, 48), (1000, 1000), (4096, 4096), (1, 1)):
        for f in (P.lf_block_linear_workspace_bytes, P.lf_block_linear_backward_workspace_bytes):
            sizes = [f(rows, outputs, inputs) for rows in (0, 1, 5, 64, 200, 1024, 4096, 16384)]
            assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes), (f, outputs, inputs, sizes)
    for cols in (7, 1024, 8192, 20000):
        sizes = [P.lf_layer_norm_workspace_bytes(rows, cols) for rows in (0, 1, 100, 511, 512, 5000)]
        assert sizes == sorted(sizes)
    assert P.lf_block_linear_workspace_bytes(-1, 8, 8) == 0 and P.lf_block_linear_backward_workspace_bytes(8, 0, 8) == 0
    assert P.lf_layer_norm_workspace_bytes(4, 0) == 0


def test_without_rows_nothing_is_enqueued():
    """No GPU is needed for that: LF_OK where a launch would fail.  Matrices without rows need no memory."""
    none = dict(data=0, scales=0)
    assert norm(rows=0, x=mat(B, 40, data=0)) == P.LF_OK
    assert save(rows=0, x=mat(B, 200, data=0), out=mat(R, 256, **none), out_t=mat(R, 0, **none)) == P.LF_OK
    assert linear(rows=0, x=mat(B, 200, data=0), x_t=mat(R, 0, **none)) == P.LF_OK
    assert distil(rows=0, top_classes=0, logits=mat(B, 40, data=0)) == P.LF_OK


def test_without_a_gpu_a_call_fails_loudly():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert [norm(), norm_back(), save(), P.lf_block_load(4, 200, mat(R, 256), mat(B, 200)), linear(), linear_back(), distil()] == [P.LF_EHIP] * 7


# ---- objects ---------------------------------------------------------------------------------------------------------------
def blocks(*shape, **kwargs):
    return on_gpu(P.E4M3Blocks(*shape, device="cpu", **kwargs))


def linear_object(*args, **kwargs):
    p = on_gpu(P.BlockLinear(*args, device="cpu", **kwargs))
    for m in (p._x_t,):
        if m is not None:
            m._gpu = GPU
    return p


def given_weights(p):
    p.set_params(blocks(p.outputs, p.inputs, tiles=True), tensor(p.outputs), blocks(p.inputs, p.outputs, tiles=True) if p._backward else None)
    return p


def test_calls_are_made_on_the_objects_gpu(calls):  # noqa: F811
    e, n = blocks(4, 200), on_gpu(P.LayerNorm(4, 40, "f32", device="cpu"))
    p, d = given_weights(linear_object(4, 8, 40, "f32", passes="backward")), on_gpu(P.Distillation(4, 40, 3, "f32", device="cpu"))
    f = given_weights(linear_object(4, 8, 40, "f32", passes="forward"))
    for current in (0, GPU):
        calls.current = current
        calls.made.clear()
        e.save(tensor(4, 200))
        e.load(out=tensor(4, 200))
        n.forward(tensor(4, 40))
        n.backward(tensor(4, 40), stored=tensor(4, 40), mean=tensor(4), rstd=tensor(4))
        f.forward(tensor(4, 40))
        p.backward(tensor(4, 8), blocks(40, 4))
        d.forward(tensor(4, 40), tensor(4, 3), tensor(4, 3, dtype=torch.int32))
        assert [c[0] for c in calls.made] == ["lf_block_save", "lf_block_load", "lf_layer_norm_forward", "lf_layer_norm_backward",
                                              "lf_block_linear_forward", "lf_block_linear_backward", "lf_distil"]
        assert all(c[1] == GPU and c[-1] == 0x1000 * GPU for c in calls.made)


def test_operands_on_the_cpu_are_refused(calls):  # noqa: F811
    x = torch.zeros(4, 40)
    e, n, d = P.E4M3Blocks(4, 40, device="cpu"), P.LayerNorm(4, 40, "f32", device="cpu"), P.Distillation(4, 40, 3, "f32", device="cpu")
    p = P.BlockLinear(4, 8, 40, "f32", device="cpu")
    for call in (lambda: e.save(x), lambda: e.load(), lambda: n.forward(x), lambda: n.backward(x, stored=x, mean=torch.zeros(4), rstd=torch.zeros(4)),
                 lambda: p.set_params(torch.zeros(8, 40)), lambda: d.forward(x, torch.zeros(4, 3), torch.zeros(4, 3, dtype=torch.int32))):
        with pytest.raises(P.LfError, match="on the CPU"):
            call()
    assert not calls.made


def test_weights_are_kept_in_8_bits_when_they_are_given_and_refreshed(calls):  # noqa: F811
    p = linear_object(4, 8, 40, "f32")
    with pytest.raises(P.LfError, match="w is NULL"):
        p.forward(tensor(4, 40))
    with pytest.raises(P.LfError, match="w is NULL"):
        p.refresh()
    w = tensor(8, 40)
    real = P.E4M3Blocks.__init__

    def on_the_gpu(self, *args, **kwargs):
        real(self, *args, **kwargs)
        self._gpu = GPU
    P.E4M3Blocks.__init__ = on_the_gpu
    try:
        p.set_params(w, tensor(8))
    finally:
        P.E4M3Blocks.__init__ = real
    assert [c[0] for c in calls.made] == ["lf_block_save"] and given(calls, 2).data == w.data_ptr()
    codes = p.w8.codes.data_ptr(), p.w8_t.codes.data_ptr()
    p.refresh()
    p.set_params(tensor(8, 40))
    assert [c[0] for c in calls.made] == ["lf_block_save"] * 3 and (p.w8.codes.data_ptr(), p.w8_t.codes.data_ptr()) == codes
    assert (given(calls, 3).data, given(calls, 4).data) == codes and given(calls, 3).type == T


def test_weights_given_in_8_bits(calls):  # noqa: F811
    p = linear_object(4, 8, 40, "f32")
    with pytest.raises(P.LfError, match="w_t"):
        p.set_params(blocks(8, 40, tiles=True))
    with pytest.raises(P.LfError, match="w_t: 40 x 8"):
        p.set_params(blocks(8, 40, tiles=True), w_t=blocks(8, 40, tiles=True))
    with pytest.raises(P.LfError, match="w_t goes with"):
        p.set_params(tensor(8, 40), w_t=blocks(40, 8, tiles=True))
    with pytest.raises(P.LfError, match="w: 8 x 40"):
        p.set_params(blocks(40, 8, tiles=True), w_t=blocks(40, 8, tiles=True))
    with pytest.raises(P.LfError, match="b: 8"):
        p.set_params(blocks(8, 40, tiles=True), tensor(40), w_t=blocks(40, 8, tiles=True))
    given_weights(p)
    p.refresh()
    assert not calls.made


def test_passes_of_fewer_rows(calls):  # noqa: F811
    p = given_weights(linear_object(300, 8, 40, "f32", z="f32", act="relu"))
    p._y, p._z, p._dx = (v.as_subclass(OnGpu) for v in (p._y, p._z, p._dx))
    x_t = p._x_t
    x_t.codes, x_t.scales = x_t.codes.as_subclass(OnGpu), x_t.scales.as_subclass(OnGpu)
    p.forward(tensor(129, 40))
    assert p.y.shape == (129, 8) and p.x_t.shape == (40, 129) and p.x_t.codes.shape == (40, 256) and p.x_t.codes.data_ptr() == x_t.codes.data_ptr()
    p.backward(tensor(129, 8))
    assert given(calls, 6).data == x_t.codes.data_ptr() and given(calls, 6).ld == 384
    with pytest.raises(P.LfError, match="x_t: 40 x 128"):
        p.backward(tensor(128, 8), z=tensor(128, 8))
    with pytest.raises(P.LfError, match="301 rows"):
        p.forward(tensor(301, 40))
    p.forward(blocks(300, 40))           # in 8 bits already: whoever made it has its transposed
    assert p.x_t is None and given(calls, 10) is None


def test_objects_check_their_tensors(calls):  # noqa: F811
    e = blocks(4, 200)
    for x in (tensor(4, 201), tensor(5, 200), tensor(4, 200).double()):
        with pytest.raises(P.LfError, match="x: 4 x 200"):
            e.save(x)
    with pytest.raises(P.LfError, match="transposed: 200 x 4"):
        e.save(tensor(4, 200), blocks(4, 200))
    with pytest.raises(P.LfError, match="codes"):
        P.E4M3Blocks.of(torch.zeros(4, 200, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), 200)
    with pytest.raises(P.LfError, match="scales"):
        P.E4M3Blocks.of(torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8), 200)
    with pytest.raises(P.LfError, match="rows"):
        P.E4M3Blocks.of(torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), 200, tiles=True)
    t = P.E4M3Blocks.of(torch.zeros(300, 256, dtype=torch.uint8), torch.zeros(3, 4, dtype=torch.uint8), 200, tiles=True)
    assert t.first(129).scales.shape == (2, 4) and t.first(300) is t and t.first_columns(7).codes.shape == (300, 128)
    assert t.first_columns(7).scales.stride(0) == 4 and t._m.type == T and t._m.scale_ld == 4
    d = on_gpu(P.Distillation(4, 40, 3, "f32", device="cpu"))
    for bad in (tensor(4, 3), tensor(4, 2, dtype=torch.int32), tensor(4, 6, dtype=torch.int32)[:, ::2], tensor(4, 3, dtype=torch.int64)):
        with pytest.raises(P.LfError, match="top_classes: 4 x 3"):
            d.forward(tensor(4, 40), tensor(4, 3), bad)
    with pytest.raises(P.LfError, match="weight: 4"):
        d.forward(tensor(4, 40), tensor(4, 3), tensor(4, 3, dtype=torch.int32), tensor(5))
    with pytest.raises(P.LfError, match="passes"):
        P.Distillation(4, 40, 3, passes="backward", device="cpu")
    with pytest.raises(P.LfError, match="activation"):
        P.BlockLinear(4, 8, 8, act="tanh", device="cpu")
    with pytest.raises(P.LfError, match="workspace"):
        P.BlockLinear(4, 8, 40, "f32", workspace=torch.zeros(8, dtype=torch.uint8), device="cpu")
    n = on_gpu(P.LayerNorm(4, 40, "f32", device="cpu"))
    with pytest.raises(P.LfError, match="shift"):
        n.shift = tensor(80)[::2]
    n.shift = tensor(40)
    n.shift.data = torch.zeros(40)
    n.forward(tensor(4, 40))
    assert n.shift.data_ptr() in calls.made[-1]
    assert on_gpu(P.Distillation(4, 40, 3, "f32", passes="forward", device="cpu")).forward(
        tensor(4, 40), tensor(4, 3), tensor(4, 3, dtype=torch.int32)).shape == (4,) and given(calls, 10) is None
