"""Trains a net of residual blocks, with its activations kept in 8 bits, to reproduce a random smooth function of its input
(synthetic data, quadratic cost), and answers single samples with the trained weights.

    python examples/train_residual_net.py [--depth 4 --width 512 --hidden 1024 --rows 512 --steps 200]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def train(depth=4, width=512, hidden=1024, rows=512, steps=200, eta=None, dtype="f32", checkpoints="e4m3", seed=0,
          say=print):
    """(cost of the first step, cost of the last, net, the target function).  eta: the descent's step; by default one that
    stays under the curvature, which grows with the values a product sums."""
    import torch

    import paper_1801_04928_amd as lf
    device = "cuda:0"
    eta = 6.4 / hidden if eta is None else eta
    net = lf.ResidualNet(depth, width, hidden, rows, dtype=dtype, checkpoints=checkpoints, device=device)
    net.init(seed)
    g = torch.Generator(device=device)
    g.manual_seed(seed + 1)
    mix = torch.randn(width, width, generator=g, device=device) * width ** -0.5

    def target(x):
        return x + torch.tanh(x.float() @ mix)

    first = last = None
    for step in range(steps):
        x = torch.randn(rows, width, generator=g, device=device).to(net.dtype)
        diff = net.forward(x).float() - target(x)
        cost = 0.5 * diff.square().sum(1).mean()            # of a sample
        net.backward((diff / rows).to(net.dtype))
        net.descend(eta)
        if step in (0, steps - 1) or step % 50 == 0:
            last = float(cost)
            first = last if first is None else first
            say(f"step {step}: cost a sample {last:.4f}", flush=True)
    return first, last, net, target


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("depth", 4), ("width", 512), ("hidden", 1024), ("rows", 512), ("steps", 200)):
        p.add_argument(f"--{name}", type=int, default=value)
    p.add_argument("--eta", type=float, default=None)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    p.add_argument("--checkpoints", choices=("e4m3", "storage"), default="e4m3")
    a = p.parse_args()
    _, _, net, target = train(a.depth, a.width, a.hidden, a.rows, a.steps, a.eta, a.dtype, a.checkpoints)
    import torch
    x = torch.randn(1, a.width, device="cuda:0").to(net.dtype)
    off = (net.forward(x).float() - target(x)).square().mean().sqrt()
    print(f"one sample: root-mean-square difference from the target {float(off):.4f}")


if __name__ == "__main__":
    main()
