"""What the operators' objects hand to the C calls (no GPU: the calls are recorded, not made)."""
import contextlib
import threading

import pytest
import torch

import paper_1801_04928_amd as P
from paper_1801_04928_amd import operators as ops

GPU = 1


class OnGpu(torch.Tensor):
    """A tensor that says it is on a GPU; its address is only handed on."""

    def get_device(self):
        return GPU


def tensor(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


class Calls:
    """Stands for the library: every entry point of the operators writes down its arguments and what is current."""

    def __init__(self):
        self.made, self.current, self.before = [], 0, lambda: None

    def __getattr__(self, name):
        real = getattr(ops.lib(), name)
        if not name.startswith("lf_") or name.endswith("_bytes") or name == "lf_operator_error":
            return real

        def call(*args):
            self.before()
            self.made.append((name, self.current, *[ops.lf_matrix.from_buffer_copy(a) if isinstance(a, ops.lf_matrix) else a
                                                    for a in args]))
            return P.LF_OK
        call.__name__ = name
        return call


@pytest.fixture
def calls(monkeypatch):
    c = Calls()
    ops._lib()          # (bound before it is replaced)
    monkeypatch.setattr(ops, "_lib", lambda: c)
    monkeypatch.setattr(ops, "_raw_stream", lambda gpu: 0x1000 * gpu)
    monkeypatch.setattr(ops, "_current_gpu", lambda: c.current, raising=False)

    @contextlib.contextmanager
    def device(gpu):
        before, c.current = c.current, gpu
        yield
        c.current = before
    monkeypatch.setattr(torch.cuda, "device", device)
    return c


def on_gpu(thing):
    """An object that was made on the CPU, as if on the GPU."""
    thing._gpu = GPU
    return thing


def linear(*args, **kwargs):
    p = on_gpu(P.Linear(*args, device="cpu", **kwargs))
    p.set_params(tensor(p.outputs, p.inputs), tensor(p.outputs))
    return p


def test_calls_are_made_on_the_objects_gpu(calls):
    """... whichever is the current one: 0 is the default stream of any."""
    e, n, p = on_gpu(P.E4M3Matrix(4, 40, device="cpu")), on_gpu(P.RmsNorm(4, 40, "f32", device="cpu")), linear(4, 8, 40, "f32")
    for current in (0, GPU):
        calls.current = current
        calls.made.clear()
        e.save(tensor(4, 40))
        e.load(out=tensor(4, 40))
        n.forward(tensor(4, 40))
        n.backward(tensor(4, 40), stored=tensor(4, 40), rstd=tensor(4))
        p.forward(tensor(4, 40))
        p.backward(tensor(4, 8), tensor(4, 40))
        assert [c[0] for c in calls.made] == ["lf_checkpoint_save", "lf_checkpoint_load", "lf_norm_forward", "lf_norm_backward",
                                              "lf_linear_forward", "lf_linear_backward"]
        assert all(c[1] == GPU and c[-1] == 0x1000 * GPU for c in calls.made)
        assert calls.current == current


def test_operands_on_the_cpu_are_refused(calls):
    """Their addresses mean nothing to a kernel."""
    x, e = torch.zeros(4, 40), P.E4M3Matrix(4, 40, device="cpu")
    n, p = P.RmsNorm(4, 40, "f32", device="cpu"), P.Linear(4, 8, 40, "f32", device="cpu")
    p.set_params(torch.zeros(8, 40))
    for call in (lambda: e.save(x), lambda: e.load(), lambda: n.forward(x), lambda: n.backward(x, stored=x, rstd=torch.zeros(4)),
                 lambda: p.forward(x), lambda: p.backward(torch.zeros(4, 8), x)):
        with pytest.raises(P.LfError, match="on the CPU"):
            call()
    assert not calls.made


def test_threads_may_load_one_matrix(calls):
    """Each call writes to its own thread's tensor, though both have theirs ready before either is made."""
    e = on_gpu(P.E4M3Matrix(4, 40, device="cpu"))
    outs = [tensor(4, 40) for _ in range(2)]
    calls.current, calls.before = GPU, threading.Barrier(2, timeout=20).wait
    threads = [threading.Thread(target=e.load, args=(out,)) for out in outs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert sorted(c[5].data for c in calls.made) == sorted(out.data_ptr() for out in outs)


def given(calls, argument):
    return calls.made[-1][2 + argument]


def test_weights_that_have_moved_are_looked_at_again(calls):
    """w, b and gain are kept by reference: a call takes them as they lie then, and refuses what no longer fits."""
    p, x = linear(4, 8, 40, "f32"), tensor(4, 40)
    for other in (torch.zeros(8, 56)[:, :40], torch.zeros(8, 40)):
        p.w.data = other
        p.forward(x)
        assert (given(calls, 4).data, given(calls, 4).ld) == (other.data_ptr(), other.stride(0))
        p.backward(tensor(4, 8), x)
        assert (given(calls, 7).data, given(calls, 7).ld) == (other.data_ptr(), other.stride(0))
    square = linear(4, 8, 8, "f32")
    n = on_gpu(P.RmsNorm(4, 40, "f32", device="cpu"))
    n.gain = tensor(40)
    for v, name, call in ((p.b, "b", lambda: p.forward(x)), (n.gain, "gain", lambda: n.forward(x))):
        v.data = torch.zeros(v.shape)
        call()
        assert v.data_ptr() in calls.made[-1]
        made = len(calls.made)
        v.data = torch.zeros(v.shape[0] - 1)
        with pytest.raises(P.LfError, match=f"{name}: "):
            call()
        assert len(calls.made) == made
    for w, why in ((torch.zeros(8, 39), "w: 8 x 40"), (torch.zeros(7, 40), "w: 8 x 40"), (torch.zeros(40, 8).t(), "contiguous")):
        p.w.data = w
        with pytest.raises(P.LfError, match=why):
            p.forward(x)
    square.w.data = square.w.data.t()          # (at the same address)
    with pytest.raises(P.LfError, match="contiguous"):
        square.forward(tensor(4, 8))
    p.w = tensor(8, 40, dtype=torch.bfloat16)
    with pytest.raises(P.LfError, match="w: torch.float32"):
        p.forward(x)


def test_what_was_kept_of_another_pass_does_not_stop_one_that_needs_none_of_it(calls):
    """Without an activation the backward pass does not look at z: neither at the last forward pass's, of other rows, nor at one given."""
    p = linear(3, 8, 40, "f32", z="f32")
    p.z = tensor(5, 8)
    p.backward(tensor(3, 8), tensor(3, 40))
    p.backward(tensor(3, 8), tensor(3, 40), z=tensor(5, 8))
    assert len(calls.made) == 2 and given(calls, 4) is None
    p = linear(3, 8, 40, "f32", z="f32", act="relu")
    p.z = tensor(5, 8)
    with pytest.raises(P.LfError, match="z: 3 x 8"):
        p.backward(tensor(3, 8), tensor(3, 40))
