"""A net of residual blocks on the operators of this package: norm, product with an activation, product, and the sum.

    block b:  s <- s + (the block before's branch),  h = norm(s),  u = act(h w1^T + b1),  branch = u w2^T + b2
    output:   s + the last branch

The addition that a block begins with is the norm's; the last one, which no norm follows, is the last product's.  What the
backward pass needs of the activations -- s, h, u and the value before the activation -- is kept in the storage type
(checkpoints="storage"), or in 8 bits ("e4m3"), half of bf16's memory.  In 8 bits h and u are only there as they are kept: the forward
products' operands are in 8 bits then, too, and the net's answers are those of 8-bit activations."""
from __future__ import annotations

from .binding import LF_EINVAL, LfError
from .operators import E4M3Matrix, Linear, RmsNorm, lf_linear_backward_workspace_bytes, lf_linear_workspace_bytes, _storage


class ResidualNet:
    """depth blocks of `width` neurons with `hidden` in between, for up to `rows` samples a pass.

    Parameters, one per block: gain (f32), w1, w2 (storage type), b1, b2 (f32); their gradients dgain, dw1, dw2, db1,
    db2.  `forward(x)` gives the output, `backward(dy)` the gradient of x."""

    def __init__(self, depth: int, width: int, hidden: int, rows: int, dtype="bf16", act: str = "gelu",
                 checkpoints="storage", device: str = "cuda:0"):
        import torch
        if depth < 1:
            raise LfError(LF_EINVAL, f"{depth} blocks")
        self.torch, self.depth, self.rows = torch, depth, rows
        self.dtype, _, dt = _storage(dtype)
        if checkpoints not in ("e4m3", "storage") and _storage(checkpoints)[0] != self.dtype:
            raise LfError(LF_EINVAL, f"checkpoints = {checkpoints!r}: e4m3, storage or the storage type's name")
        kept = "e4m3" if checkpoints == "e4m3" else self.dtype
        new = dict(dtype=self.dtype, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        # what the next block overwrites: the running sum, a branch, the gradients on their way down
        self._s, self._branch, self._ds, self._du, self._dh = (
            torch.empty((rows, n), **new) for n in (width, width, width, hidden, width))
        nbytes = max(f(rows, o, i, dt) for f in (lf_linear_workspace_bytes, lf_linear_backward_workspace_bytes)
                     for o, i in ((hidden, width), (width, hidden)))
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.out = torch.empty((rows, width), **new)
        self.norms, self.ups, self.downs, self._sums = [], [], [], []
        self.w1, self.b1, self.w2, self.b2 = [], [], [], []
        for b in range(depth):
            last = b == depth - 1
            # the running sum is updated in place; its checkpoint, or in the storage type the sum itself, is the block's
            self._sums.append(E4M3Matrix(rows, width, device) if kept == "e4m3" else torch.empty((rows, width), **new))
            self.norms.append(RmsNorm(rows, width, dtype, out=kept, sum=self._s if kept == "e4m3" else self._sums[b],
                                      dx=self._ds, device=device))
            self.ups.append(Linear(rows, hidden, width, dtype, act=act, y=kept, z=kept if act != "none" else "none",
                                   dx=self._dh, workspace=scratch, device=device))
            self.downs.append(Linear(rows, width, hidden, dtype, y=self.out if last else self._branch, dx=self._du,
                                     workspace=scratch, device=device))
            self.w1.append(torch.empty((hidden, width), **new))
            self.b1.append(torch.zeros(hidden, **f32))
            self.w2.append(torch.empty((width, hidden), **new))
            self.b2.append(torch.zeros(width, **f32))
            self.ups[b].set_params(self.w1[b], self.b1[b])
            self.downs[b].set_params(self.w2[b], self.b2[b])
        self._masters = None
        self.gain = [n.gain for n in self.norms]
        self.dgain = [n.dgain for n in self.norms]
        self.dw1, self.db1 = [p.dw for p in self.ups], [p.db for p in self.ups]
        self.dw2, self.db2 = [p.dw for p in self.downs], [p.db for p in self.downs]

    def init(self, seed: int = 0) -> None:
        """Random weights: variance 1 / fan-in, the second product's divided by the depth, so that the sum grows little."""
        g = self.torch.Generator(device=self.w1[0].device)
        g.manual_seed(seed)
        for w1, w2 in zip(self.w1, self.w2):
            for w, scale in ((w1, 1.0), (w2, self.depth ** -0.5)):
                v = self.torch.randn(w.shape, generator=g, device=w.device)
                w.copy_(v * (scale * w.shape[1] ** -0.5))

    def forward(self, x):
        s, branch = x, None
        for b in range(self.depth):
            h = self.norms[b].forward(s, branch)
            s = self.norms[b].sum
            if isinstance(self._sums[b], E4M3Matrix):
                self._sums[b].first(x.shape[0]).save(s)
            u = self.ups[b].forward(h)
            branch = self.downs[b].forward(u, residual=s if b == self.depth - 1 else None)
        return branch

    def backward(self, dy):
        n, ds = dy.shape[0], dy
        for b in reversed(range(self.depth)):
            du = self.downs[b].backward(ds, self.ups[b].y)
            dh = self.ups[b].backward(du, self.norms[b].y)
            kept = self._sums[b]
            ds = self.norms[b].backward(dh, ds, stored=kept.first(n) if isinstance(kept, E4M3Matrix) else kept[:n])
        return ds

    def descend(self, eta: float) -> None:
        """A plain gradient-descent step: every parameter less eta times its gradient.  Weights in bf16 descend in fp32 copies, made
        in the first step, and are these copies' roundings, so that steps smaller than half of bf16's add up.  A weight that was
        set to something else meanwhile goes on from there."""
        torch = self.torch
        if self.dtype == torch.float32:
            weights = [*self.w1, *self.w2]
        else:
            if self._masters is None:
                self._masters = [w.float() for w in (*self.w1, *self.w2)]
            weights = self._masters
            for w, master in zip((*self.w1, *self.w2), weights):
                master.copy_(torch.where(master.to(w.dtype) == w, master, w.float()))
        for p, g in zip((*weights, *self.b1, *self.b2, *self.gain), (*self.dw1, *self.dw2, *self.db1, *self.db2, *self.dgain)):
            p.add_(g, alpha=-eta)
        for w, master in zip((*self.w1, *self.w2), weights):
            if master is not w:
                w.copy_(master)
