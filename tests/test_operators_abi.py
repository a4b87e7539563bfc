"""Host-side checks of the residual blocks' operators (no GPU): every symbol that lf_operators.h declares is exported and
bound, arguments are refused before anything is enqueued, and workspaces that serve some rows serve fewer."""
import ctypes as C
import os
import re

import pytest

import paper_1801_04928_amd as P
from paper_1801_04928_amd import operators as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20          # a "device pointer" that is only checked for alignment
F, B, E = P.LF_MATRIX_F32, P.LF_MATRIX_BF16, P.LF_MATRIX_E4M3


def mat(kind, ld, data=FAKE, scales=FAKE, scale_ld=None):
    return P.lf_matrix(data, ld, scales if kind == E else None, scale_ld if scale_ld is not None else -(-ld // 32), kind)


def declared():
    text = open(os.path.join(ROOT, "include", "lf_operators.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(lf_\w+)\s*\(", text)))


def test_every_declared_symbol_is_exported_and_bound():
    names = declared()
    assert {"lf_norm_forward", "lf_linear_backward", "lf_checkpoint_save", "lf_operator_error"} <= set(names)
    for name in names:
        assert hasattr(P.lib(), name), name
        assert callable(getattr(P, name)), name


def test_matrix_layout_is_the_headers():
    assert C.sizeof(P.lf_matrix) == 40
    assert [getattr(P.lf_matrix, n).offset for n in ("data", "ld", "scales", "scale_ld", "type")] == [0, 8, 16, 24, 32]


def save(rows=4, cols=40, x=mat(B, 40), out=mat(E, 64)):
    return P.lf_checkpoint_save(rows, cols, x, out)


@pytest.mark.parametrize("change, status, word", [
    (dict(rows=-1), P.LF_EINVAL, "rows"), (dict(cols=0), P.LF_EINVAL, "cols"),
    (dict(rows=(1 << 28) + 1), P.LF_EUNSUPPORTED, "rows"), (dict(cols=1 << 22), P.LF_EUNSUPPORTED, "cols"),
    (dict(x=None), P.LF_EINVAL, "NULL"), (dict(x=mat(E, 64)), P.LF_EINVAL, "type"), (dict(x=mat(7, 64)), P.LF_EINVAL, "type"),
    (dict(x=mat(B, 39)), P.LF_EINVAL, "ld"), (dict(x=mat(B, 40, data=0)), P.LF_EINVAL, "NULL"),
    (dict(x=mat(B, 40, data=FAKE + 1)), P.LF_EINVAL, "misaligned"), (dict(x=mat(F, 40, data=FAKE + 2)), P.LF_EINVAL, "misaligned"),
    (dict(x=mat(B, (4 << 20) + 1)), P.LF_EUNSUPPORTED, "ld"),
    (dict(out=mat(B, 40)), P.LF_EINVAL, "type"), (dict(out=mat(E, 32)), P.LF_EINVAL, "ld"), (dict(out=mat(E, 80)), P.LF_EINVAL, "32"),
    (dict(out=mat(E, 64, data=FAKE + 8)), P.LF_EINVAL, "misaligned"), (dict(out=mat(E, 64, scales=0)), P.LF_EINVAL, "scales"),
    (dict(out=mat(E, 64, scale_ld=1)), P.LF_EINVAL, "scale_ld")])
def test_checkpoint_refusals(change, status, word):
    assert save(**change) == status
    assert word in P.lf_operator_error() and "lf_checkpoint_save" in P.lf_operator_error()


def test_checkpoint_load_refusals():
    assert P.lf_checkpoint_load(4, 40, mat(B, 40), mat(B, 40)) == P.LF_EINVAL
    assert P.lf_checkpoint_load(4, 40, mat(E, 64), mat(E, 64)) == P.LF_EINVAL
    assert P.lf_checkpoint_load(4, 40, mat(E, 64), None) == P.LF_EINVAL


def norm(rows=4, cols=40, x=mat(B, 40), branch=None, gain=FAKE, eps=1e-6, total=mat(B, 40), y=mat(E, 64), rstd=FAKE):
    return P.lf_norm_forward(rows, cols, x, branch, gain, eps, total, y, rstd)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(cols=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(x=mat(E, 64)),
    dict(branch=mat(F, 40)), dict(branch=mat(B, 39)), dict(gain=FAKE + 2), dict(total=mat(E, 64)), dict(total=mat(F, 40)),
    dict(y=None), dict(y=mat(F, 40)), dict(y=mat(E, 40)), dict(rstd=FAKE + 1)])
def test_norm_forward_refusals(change):
    assert norm(**change) == P.LF_EINVAL
    assert "lf_norm_forward" in P.lf_operator_error()


def norm_back(rows=4, cols=40, dy=mat(B, 40), total=mat(E, 64), gain=FAKE, rstd=FAKE, dsum=None, dx=mat(B, 40), dgain=FAKE,
              workspace=FAKE, nbytes=1 << 20):
    return P.lf_norm_backward(rows, cols, dy, total, gain, rstd, dsum, dx, dgain, workspace, nbytes)


@pytest.mark.parametrize("change", [
    dict(dy=None), dict(dy=mat(E, 64)), dict(total=None), dict(total=mat(F, 40)), dict(gain=FAKE + 2), dict(rstd=0), dict(rstd=FAKE + 2),
    dict(dsum=mat(F, 40)), dict(dx=None), dict(dx=mat(F, 40)), dict(dx=mat(E, 64)), dict(dgain=FAKE + 1), dict(workspace=0),
    dict(workspace=FAKE + 16), dict(nbytes=0)])
def test_norm_backward_refusals(change):
    assert norm_back(**change) == P.LF_EINVAL
    assert "lf_norm_backward" in P.lf_operator_error()


def linear(rows=4, outputs=48, inputs=40, x=mat(E, 64), w=mat(B, 40), bias=FAKE, act=P.LF_ACT_GELU, residual=None,
           y=mat(B, 48), z=mat(E, 64), workspace=FAKE, nbytes=1 << 30):
    return P.lf_linear_forward(rows, outputs, inputs, x, w, bias, act, residual, y, z, workspace, nbytes)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(outputs=0), dict(inputs=0), dict(x=None), dict(x=mat(F, 40)), dict(x=mat(E, 32)), dict(w=None),
    dict(w=mat(E, 64)), dict(w=mat(B, 39)), dict(bias=FAKE + 2), dict(act=5), dict(act=-1), dict(residual=mat(F, 48)),
    dict(residual=mat(E, 64)), dict(y=None), dict(y=mat(F, 48)), dict(y=mat(E, 48)), dict(z=mat(F, 48)), dict(z=mat(B, 47))])
def test_linear_forward_refusals(change):
    assert linear(**change) == P.LF_EINVAL
    assert "lf_linear_forward" in P.lf_operator_error()


def test_linear_forward_asks_for_its_workspace():
    # a long contraction of few tiles is split: its partial sums need scratch
    need = P.lf_linear_workspace_bytes(4, 48, 8192, P.LF_BF16)
    assert need > 0 and need % 256 == 0
    args = dict(inputs=8192, x=mat(B, 8192), w=mat(B, 8192))
    assert linear(**args, nbytes=need - 1) == P.LF_EINVAL and "workspace" in P.lf_operator_error()
    assert linear(**args, workspace=0, nbytes=need) == P.LF_EINVAL
    assert linear(**args, workspace=FAKE + 128, nbytes=need) == P.LF_EINVAL


def linear_back(rows=4, outputs=48, inputs=40, dy=mat(B, 48), z=mat(E, 64), act=P.LF_ACT_SILU, x=mat(E, 64), w=mat(B, 40),
                dx=mat(B, 40), dw=mat(F, 40), db=FAKE, workspace=FAKE, nbytes=1 << 30):
    return P.lf_linear_backward(rows, outputs, inputs, dy, z, act, x, w, dx, dw, db, workspace, nbytes)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(outputs=0), dict(inputs=0), dict(dy=None), dict(dy=mat(E, 64)), dict(z=None), dict(z=mat(F, 48)),
    dict(act=9), dict(x=None), dict(x=mat(F, 40)), dict(w=None), dict(w=mat(F, 40)), dict(w=mat(E, 64)), dict(dx=mat(F, 40)),
    dict(dw=mat(E, 64)), dict(dw=mat(B, 39)), dict(db=FAKE + 2), dict(workspace=0), dict(nbytes=64)])
def test_linear_backward_refusals(change):
    assert linear_back(**change) == P.LF_EINVAL
    assert "lf_linear_backward" in P.lf_operator_error()


def test_workspaces_serve_fewer_rows():
    for dt in (P.LF_F32, P.LF_BF16):
        for outputs, inputs in ((48, 8192), (8192, 48), (1000, 1000), (4096, 4096), (1, 1)):
            for f in (P.lf_linear_workspace_bytes, P.lf_linear_backward_workspace_bytes):
                sizes = [f(rows, outputs, inputs, dt) for rows in (0, 1, 5, 64, 200, 1024, 4096, 16384)]
                assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes), (f, outputs, inputs, sizes)
    sizes = [P.lf_norm_workspace_bytes(rows, 8192) for rows in (0, 1, 100, 511, 512, 5000)]
    assert sizes == sorted(sizes)
    assert P.lf_linear_workspace_bytes(-1, 8, 8, P.LF_F32) == 0 and P.lf_linear_workspace_bytes(8, 8, 8, 2) == 0
    assert P.lf_norm_workspace_bytes(4, 0) == 0


def test_without_rows_nothing_is_enqueued():
    """No GPU is needed for that: LF_OK where a launch would fail.  Matrices without rows need no memory."""
    empty = dict(x=mat(B, 40, data=0))
    assert P.lf_checkpoint_save(0, 40, mat(B, 40, data=0), mat(E, 64, data=0, scales=0)) == P.LF_OK
    assert norm(rows=0, **empty) == P.LF_OK
    assert linear(rows=0, x=mat(E, 64, data=0, scales=0)) == P.LF_OK


def test_without_a_gpu_a_call_fails_loudly():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert save() == P.LF_EHIP and P.lf_operator_error()
    assert norm() == P.LF_EHIP and norm_back() == P.LF_EHIP
    assert linear() == P.LF_EHIP and linear_back() == P.LF_EHIP


def test_errors_are_the_threads_own():
    import threading
    assert save(rows=-1) == P.LF_EINVAL
    seen = []

    def other():
        seen.append(P.lf_operator_error())
        norm(eps=-1.0)
        seen.append(P.lf_operator_error())
    t = threading.Thread(target=other)
    t.start()
    t.join()
    assert seen[0] == "no error" and "eps" in seen[1] and "rows" in P.lf_operator_error()


def test_objects_check_their_tensors():
    import torch
    x, e = torch.zeros(4, 40), P.E4M3Matrix(4, 40, device="cpu")
    with pytest.raises(P.LfError, match="x: 4 x 40"):
        e.save(x.double())
    with pytest.raises(P.LfError, match="x: 4 x 40"):
        e.save(torch.zeros(5, 40))
    with pytest.raises(P.LfError, match="x: 4 x 40"):
        e.save(torch.zeros(160))
    with pytest.raises(P.LfError, match="contiguous"):
        e.save(torch.zeros(40, 4).t())
    with pytest.raises(P.LfError, match="x: 4 x 40"):
        P.RmsNorm(4, 40, "f32", device="cpu").forward(P.E4M3Matrix(4, 41, device="cpu"))
    with pytest.raises(P.LfError, match="gain"):
        n = P.RmsNorm(4, 40, "f32", device="cpu")
        n.gain = torch.zeros(80)[::2]
        n.forward(x)
    p = P.Linear(4, 8, 40, "f32", device="cpu")
    with pytest.raises(P.LfError, match="w: torch.float32"):
        p.set_params(torch.zeros(8, 40, dtype=torch.bfloat16))
    with pytest.raises(P.LfError, match="b: 8"):
        p.set_params(torch.zeros(8, 40), torch.zeros(40))
    with pytest.raises(P.LfError, match="w is NULL"):
        p.forward(x)
    with pytest.raises(P.LfError, match="workspace"):
        P.Linear(4, 8, 40, "f32", workspace=torch.zeros(8, dtype=torch.uint8), device="cpu")
    m = ops._matrix("x", torch.zeros(4, 64)[1:2, 1:41], (1, 40), -1, P.lf_matrix())
    assert m.ld >= 40 and m.type == F
    with pytest.raises(P.LfError, match="codes"):
        P.E4M3Matrix.of(torch.zeros(4, 40, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8), 40)
    with pytest.raises(P.LfError, match="scales"):
        P.E4M3Matrix.of(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8), 40)
    e = P.E4M3Matrix.of(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8), 40)
    assert e.first(2).shape == (2, 40) and e.first(4) is e
    with pytest.raises(P.LfError, match="activation"):
        P.Linear(4, 8, 8, act="tanh", device="cpu")
    with pytest.raises(P.LfError, match="storage type"):
        P.RmsNorm(4, 8, dtype=torch.float16, device="cpu")
    with pytest.raises(P.LfError, match="passes"):
        P.RmsNorm(4, 8, passes="none", device="cpu")
