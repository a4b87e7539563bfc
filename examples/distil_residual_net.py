"""A student net learns from a teacher's top logits (synthetic data): layer norms, products in 8 bits with blocks of 128, the distillation
loss; then the student answers single samples.

    python examples/distil_residual_net.py [--depth 2 --width 256 --hidden 512 --classes 1000 --top 16 --rows 512 --steps 100]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def distil(depth=2, width=256, hidden=512, classes=1000, top=16, rows=512, steps=100, eta=0.5, temperature=2.0, dtype="bf16",
           checkpoints="storage", seed=0, say=print):
    """(loss of the first step, loss of the last, student, teacher)."""
    import torch

    import paper_1801_04928_amd as lf
    device = "cuda:0"
    teacher = lf.ResidualNet(2 * depth, width, hidden, rows, dtype=dtype, classes=classes, passes="forward", device=device)
    teacher.init(seed)
    teacher.w_out.mul_(3)                                   # a teacher that is sure of something
    student = lf.ResidualNet(depth, width, hidden, rows, dtype=dtype, checkpoints=checkpoints, norm="layer", products="e4m3_128",
                             classes=classes, device=device)
    student.init(seed + 1)
    g = torch.Generator(device=device)
    g.manual_seed(seed + 2)
    weight = torch.full((rows,), 1.0 / rows, device=device)
    first = last = None
    for step in range(steps):
        x = torch.randn(rows, width, generator=g, device=device).to(student.dtype)
        logits, which = torch.topk(teacher.forward(x).float(), top, dim=1)
        loss = student.distil(x, logits, which.to(torch.int32), temperature, weight)
        student.descend(eta)
        if step in (0, steps - 1) or step % 25 == 0:
            last = float(loss.sum())
            first = last if first is None else first
            say(f"step {step}: loss a sample {last:.4f}", flush=True)
    return first, last, student, teacher


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("depth", 2), ("width", 256), ("hidden", 512), ("classes", 1000), ("top", 16), ("rows", 512), ("steps", 100)):
        p.add_argument(f"--{name}", type=int, default=value)
    p.add_argument("--eta", type=float, default=0.5)
    p.add_argument("--temperature", type=float, default=2.0)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    p.add_argument("--checkpoints", choices=("e4m3", "storage"), default="storage")
    a = p.parse_args()
    _, _, student, teacher = distil(a.depth, a.width, a.hidden, a.classes, a.top, a.rows, a.steps, a.eta, a.temperature, a.dtype, a.checkpoints)
    import torch
    x = torch.randn(1, a.width, device="cuda:0").to(student.dtype)
    theirs = int(teacher.forward(x).float().argmax())
    order = student.forward(x).float().argsort(descending=True)[0].tolist()
    print(f"one sample: the teacher's class is the student's number {1 + order.index(theirs)}")


if __name__ == "__main__":
    main()
