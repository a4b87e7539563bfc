"""ResidualNet in HIP graphs: passes and steps that are captured and replayed among the program's own work give what the same calls give
one by one, bit for bit."""
import pytest
import torch

import paper_1801_04928_amd as P
from tests.student_util import DEV, TYPE, values

pytestmark = pytest.mark.gpu
ROWS, WIDTH, HIDDEN, CLASSES, TOP, T, ETA = 20, 40, 136, 45, 4, 2.0, 2.0 ** -7
KINDS = [("f32", "storage"), ("bf16", "storage"), ("f32", "e4m3_128"), ("bf16", "e4m3_128")]


def net(dtype, products):
    n = P.ResidualNet(2, WIDTH, HIDDEN, ROWS, dtype=dtype, norm="layer", products=products, classes=CLASSES)
    n.init(3)
    return n


def batch(seed, dtype):
    order = torch.argsort(values(seed, ROWS, CLASSES), 1)[:, :TOP].to(torch.int32)
    return values(seed + 1, ROWS, WIDTH).to(TYPE[dtype]).to(DEV), values(seed + 2, ROWS, TOP, std=2).float().to(DEV), order.to(DEV)


def captured(call):
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = call()
    torch.cuda.synchronize()
    return graph, out


def step(n, data):
    loss = n.distil(*data, T)
    n.descend(ETA)
    return loss


def parameters(n):
    return [*n.w1, *n.w2, n.w_out, *n.b1, *n.b2, n.b_out, *n.gain, *n.shift]


def same_nets(a, b):
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(parameters(a), parameters(b)))


@pytest.mark.parametrize("before", ["nothing", "forward", "step"])
@pytest.mark.parametrize("dtype, products", KINDS)
def test_captured_steps_are_the_eager_ones(dtype, products, before):
    """(Steps so small that weights in bf16 would not see one of them.)"""
    mine, eager, data = net(dtype, products), net(dtype, products), batch(0, dtype)
    for n in (mine, eager):
        if before == "forward":
            n.forward(data[0])
        elif before == "step":
            step(n, data)
    graph, loss = captured(lambda: step(mine, data))
    x = batch(50, dtype)[0]
    for k in range(4):
        for to, new in zip(data, batch(10 * k, dtype)):
            to.copy_(new)
        graph.replay()
        assert torch.equal(loss, step(eager, data))
        same_nets(mine, eager)
        if k % 2:                                              # eager work between replays is of the weights as they are now
            assert torch.equal(mine.forward(x), eager.forward(x))
    assert not torch.equal(mine.w1[0], net(dtype, products).w1[0])
    assert torch.equal(step(mine, data), step(eager, data))
    same_nets(mine, eager)
    assert torch.equal(mine.forward(x), eager.forward(x))


@pytest.mark.parametrize("dtype, products", KINDS)
def test_a_captured_pass_follows_eager_steps(dtype, products):
    mine, eager, data = net(dtype, products), net(dtype, products), batch(0, dtype)
    mine.forward(data[0])
    forward, y = captured(lambda: mine.forward(data[0]))
    distil, loss = captured(lambda: mine.distil(*data, T))
    for k in range(3):
        distil.replay()
        want = step(eager, data)
        assert torch.equal(loss, want)
        mine.descend(ETA)
        forward.replay()
        assert torch.equal(y, eager.forward(data[0]))
    for n in (mine, eager):
        n.init(5)
    forward.replay()
    assert torch.equal(y, eager.forward(data[0]))
    for n in (mine, eager):
        n.w1[0].mul_(0.5)
        n.refresh()
    forward.replay()
    assert torch.equal(y, eager.forward(data[0]))


@pytest.mark.parametrize("before", ["nothing", "forward"])
@pytest.mark.parametrize("dtype, products", KINDS)
def test_an_eager_pass_follows_captured_steps(dtype, products, before):
    mine, eager, data = net(dtype, products), net(dtype, products), batch(0, dtype)
    if before == "forward":
        mine.forward(data[0])
    # (gradients to descend by, which no pass has left yet)
    for n in (mine, eager):
        for g in (*n.dw1, *n.dw2, n.dw_out, *n.db1, *n.db2, n.db_out, *n.dgain, *n.dshift):
            g.fill_(0.25)
    descend, _ = captured(lambda: mine.descend(ETA))
    forward, y = captured(lambda: mine.forward(data[0]))
    # a pass that was captured has not run: an eager one finds nothing done
    assert torch.equal(mine.forward(data[0]), eager.forward(data[0]))
    for k in range(3):
        descend.replay()
        eager.descend(ETA)
        same_nets(mine, eager)
        want = eager.forward(data[0])
        assert torch.equal(mine.forward(data[0]), want)
        y.zero_()
        forward.replay()
        assert torch.equal(y, want)


@pytest.mark.parametrize("dtype, products", KINDS)
def test_weights_that_are_set_behind_an_eager_step_are_the_next_pass_s(dtype, products):
    """... whether or not a pass was captured."""
    mine, eager, data = net(dtype, products), net(dtype, products), batch(0, dtype)
    mine.forward(data[0])
    graph, y = captured(lambda: mine.forward(data[0]))
    for k in range(2):
        for n in (mine, eager):
            step(n, data)
            n.w2[1].mul_(0.5)
        assert torch.equal(mine.forward(data[0]), eager.forward(data[0]))
        graph.replay()
        assert torch.equal(y, eager.forward(data[0]))
        same_nets(mine, eager)
