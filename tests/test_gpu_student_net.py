"""The student nets' operators together: ResidualNet with layer norms, products in blocks of 128 and the distillation loss, and its example."""
import importlib.util
import os
import sys

import pytest
import torch

import paper_1801_04928_amd as P
from tests import student_reference as R
from tests.student_util import DEV, TYPE, values

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def teacher_of(rows, classes, top, seed=7):
    order = torch.argsort(values(seed, rows, classes), 1)[:, :top].to(torch.int32)
    return values(seed + 1, rows, top, std=2), order, values(seed + 2, rows).abs().float().double()


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_gradients_of_the_whole_net(norm):
    """fp32 against torch's gradients in 64 bits.  Every operator is off by at most (n + 40) u of sums of magnitudes, n <= 70, 7e-6; sums of random
    signs are a tenth of their magnitudes, and some ten operators follow each other: 1e-3 of a gradient's norm covers it."""
    rows, width, hidden, classes, top, T = 33, 40, 70, 50, 6, 2.0
    net = P.ResidualNet(2, width, hidden, rows, dtype="f32", norm=norm, classes=classes)
    net.init(3)
    for k, v in enumerate((*net.gain, *net.shift, *net.b1, *net.b2, net.b_out)):
        v.add_(values(k, v.shape[0], std=0.2).float().to(DEV))
    x, (t, order, weight) = values(1, rows, width), teacher_of(rows, classes, top)
    loss = net.distil(x.float().to(DEV), t.float().to(DEV), order.to(DEV), T, weight.float().to(DEV)).double().cpu()

    def leaf(v):
        return v.detach().double().cpu().requires_grad_()
    p = {k: [leaf(v) for v in vs] for k, vs in dict(w1=net.w1, w2=net.w2, b1=net.b1, b2=net.b2, gain=net.gain, shift=net.shift, out=[net.w_out, net.b_out]).items()}

    def normed(s, b):
        if norm == "rms":
            return s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * p["gain"][b]
        off = s - s.mean(1, keepdim=True)
        return off * (off.square().mean(1, keepdim=True) + 1e-5).rsqrt() * p["gain"][b] + p["shift"][b]
    s = x
    for b in range(2):
        s = s + R.act(normed(s, b) @ p["w1"][b].t() + p["b1"][b], "gelu") @ p["w2"][b].t() + p["b2"][b]
    z = normed(s, 2) @ p["out"][0].t() + p["out"][1]
    log_p, log_q = torch.log_softmax(t / T, 1), torch.log_softmax(z / T, 1).gather(1, order.long())
    want = weight * T * T * (log_p.exp() * (log_p - log_q)).sum(1)
    want.sum().backward()
    assert float((loss - want.detach()).norm() / want.detach().norm()) < 1e-3
    pairs = [*zip((*net.dw1, *net.dw2, *net.db1, *net.db2, *net.dgain, *net.dshift, net.dw_out, net.db_out),
                  (*p["w1"], *p["w2"], *p["b1"], *p["b2"], *p["gain"], *p["shift"], *p["out"]))]
    assert len(pairs) == 13 + (3 if norm == "layer" else 0)
    for k, (got, of) in enumerate(pairs):
        assert float((got.double().cpu() - of.grad).norm() / of.grad.norm()) < 1e-3, k


@pytest.mark.parametrize("checkpoints", ["storage", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_pass_is_its_operators(dtype, checkpoints):
    """A whole pass of learning, bit for bit what the operators give that are called one by one."""
    rows, width, hidden, classes, top, n = 140, 72, 150, 133, 5, 131
    net = P.ResidualNet(2, width, hidden, rows, dtype=dtype, act="silu", checkpoints=checkpoints, norm="layer", products="e4m3_128", classes=classes)
    net.init(5)
    for k, v in enumerate((*net.shift, *net.b1, *net.b2, net.b_out)):
        v.add_(values(k, v.shape[0], std=0.2).float().to(DEV))
    kind = TYPE[dtype]
    x, (t, order, weight) = values(1, n, width).to(kind).to(DEV), teacher_of(n, classes, top)
    t, order, weight = t.float().to(DEV), order.to(DEV), weight.float().to(DEV)
    for step in range(2):
        weights = [w.clone() for w in (*net.w1, *net.w2, net.w_out)]
        vectors = [v.clone() for v in (*net.b1, *net.b2, net.b_out)]
        products = []
        for k, (w, b) in enumerate(zip(weights, vectors)):
            p = P.BlockLinear(n, *w.shape, dtype, act="silu" if k < 2 else "none", z=("e4m3_128" if checkpoints == "e4m3" else dtype) if k < 2 else "none")
            p.set_params(w, b)
            products.append(p)
        ups, downs, head = products[:2], products[2:4], products[4]
        norms = [P.LayerNorm(n, width, dtype) for _ in range(3)]
        for m, gain, shift in zip(norms, net.gain, net.shift):
            m.gain, m.shift = gain.clone(), shift.clone()
        s, branch, kept = x, None, []
        for b in range(3):
            h = norms[b].forward(s, branch)
            s = norms[b].sum
            kept.append(P.E4M3Matrix(n, width).save(s) if checkpoints == "e4m3" else s)
            if b < 2:
                branch = downs[b].forward(ups[b].forward(h))
        logits = head.forward(h)
        loss = P.Distillation(n, classes, top, dtype, temperature=2.0)
        want = loss.forward(logits, t, order, weight)
        ds = norms[2].backward(head.backward(loss.dlogits), stored=kept[2]).clone()
        for b in (1, 0):
            ds = norms[b].backward(ups[b].backward(downs[b].backward(ds)), ds, stored=kept[b]).clone()

        assert torch.equal(net.distil(x, t, order, 2.0, weight), want) and torch.equal(net._ds[:n], ds)
        for got, all_ in ((net.dw1, ups), (net.dw2, downs), ([net.dw_out], [head])):
            assert all(torch.equal(g, p.dw) for g, p in zip(got, all_))
        for got, all_ in ((net.db1, ups), (net.db2, downs), ([net.db_out], [head])):
            assert all(torch.equal(g, p.db) for g, p in zip(got, all_))
        assert all(torch.equal(g, m.dgain) and torch.equal(d, m.dshift) for g, d, m in zip(net.dgain, net.dshift, norms))
        net.descend(0.25)          # the second pass is of other weights
        assert not torch.equal(net.w1[0], weights[0])


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("classes", [None, 45])
def test_a_net_for_answers_answers_as_the_one_that_learns(norm, classes):
    nets = [P.ResidualNet(2, 40, 136, 20, dtype="f32", norm=norm, classes=classes, passes=passes) for passes in ("both", "forward")]
    x = values(1, 20, 40).float().to(DEV)
    for net in nets:
        net.init(2)
    answers = [net.forward(x[:n]).clone() for net in nets for n in (20, 1)]
    assert torch.equal(answers[0], answers[2]) and torch.equal(answers[1], answers[3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("classes", [None, 45])
def test_a_net_for_answers_is_its_operators(norm, classes, dtype):
    """In blocks of 128 the norm and the first product write the next one's operand: bit for bit what the operators give.  The net that learns rounds
    to the storage type before it keeps them: every value of an operand is off by a code at most, 2^-3 of it, so the answers' norm by 2^-2."""
    nets = [P.ResidualNet(2, 40, 136, 20, dtype=dtype, norm=norm, products="e4m3_128", classes=classes, passes=passes) for passes in ("both", "forward")]
    for net in nets:
        net.init(2)
    net = nets[1]
    for n in (20, 1):
        x = values(1, 20, 40).to(TYPE[dtype]).to(DEV)[:n]
        norms = [P.LayerNorm(n, 40, dtype, out="e4m3_128", passes="forward") if norm == "layer" else P.RmsNorm(n, 40, dtype, passes="forward") for _ in range(3)]

        def product(w, **kwargs):
            p = P.BlockLinear(n, *w.shape, dtype, passes="forward", **kwargs)
            p.set_params(w, torch.zeros(w.shape[0], device=DEV))
            return p
        s, branch = x, None
        for b in range(2):
            h = norms[b].forward(s, branch)
            s = norms[b].sum
            u = product(net.w1[b], act="gelu", y="e4m3_128").forward(h)
            branch = product(net.w2[b]).forward(u, residual=s if b == 1 and classes is None else None)
        want = branch if classes is None else product(net.w_out).forward(norms[2].forward(s, branch))
        got = net.forward(x)
        assert torch.equal(got, want)
        other = nets[0].forward(x).float()
        assert float((got.float() - other).norm() / other.norm()) < 2.0 ** -2


def test_a_pass_of_no_rows():
    net = P.ResidualNet(2, 40, 24, 4, norm="layer", products="e4m3_128", classes=9)
    net.init()
    grads = [*net.dw1, *net.dw2, *net.db1, *net.db2, *net.dgain, *net.dshift, net.dw_out, net.db_out]
    for g in grads:
        g.fill_(7.0)
    x = torch.ones(4, 40, dtype=torch.bfloat16, device=DEV)[:0]
    assert net.distil(x, torch.zeros(0, 3, device=DEV), torch.zeros(0, 3, dtype=torch.int32, device=DEV)).shape == (0,)
    assert all(bool((g == 0).all()) for g in grads)


@pytest.mark.parametrize("checkpoints", ["e4m3", "storage"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_example_takes_its_options(dtype, checkpoints, monkeypatch, capsys):
    spec = importlib.util.spec_from_file_location("distil_residual_net", os.path.join(ROOT, "examples", "distil_residual_net.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    monkeypatch.setattr(sys, "argv", ["distil_residual_net.py", "--depth", "1", "--width", "64", "--hidden", "72", "--classes", "50", "--top", "5",
                                      "--rows", "32", "--steps", "3", "--dtype", dtype, "--checkpoints", checkpoints])
    module.main()
    out = capsys.readouterr().out
    assert "step 2: loss" in out and "one sample" in out
