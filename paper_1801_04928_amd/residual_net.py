"""A net of residual blocks on the operators of this package: norm, product with an activation, product, and the sum.

    block b:  s <- s + (the block before's branch),  h = norm(s),  u = act(h w1^T + b1),  branch = u w2^T + b2
    output:   s + the last branch, or with classes the logits  norm(s + the last branch) w_out^T + b_out

The addition that a block begins with is the norm's; the last one, which no norm follows, is the last product's.  What the
backward pass needs of the activations -- s, h, u and the value before the activation -- is kept in the storage type
(checkpoints="storage"), or in 8 bits ("e4m3"), half of bf16's memory.  In 8 bits h and u are only there as they are kept: the forward
products' operands are in 8 bits then, too, and the net's answers are those of 8-bit activations.

With products="e4m3_128" all products, the backward pass's too, are of operands in 8 bits with blocks of 128; of h and u the backward
pass keeps the transposed codes then, whatever `checkpoints` says of s and of the value before the activation."""
from __future__ import annotations

from .binding import LF_EINVAL, LfError
from .operators import (BlockLinear, Distillation, E4M3Blocks, E4M3Matrix, LayerNorm, Linear, RmsNorm, lf_block_linear_backward_workspace_bytes,
                        lf_block_linear_workspace_bytes, lf_linear_backward_workspace_bytes, lf_linear_workspace_bytes, _storage)


class ResidualNet:
    """depth blocks of `width` neurons with `hidden` in between, for up to `rows` samples a pass.

    norm: "rms", or "layer", the layer norm.  products: "storage", or "e4m3_128", in 8 bits with blocks of 128.  classes: logits of so
    many classes come out, by a norm and a product of their own.  passes: "both", or "forward" for answers alone.

    Parameters, one per block: gain (f32), with norm="layer" shift (f32), w1, w2 (storage type), b1, b2 (f32); with classes
    another gain (and shift), w_out and b_out.  Their gradients: dgain, dshift, dw1, dw2, db1, db2, dw_out, db_out.  `forward(x)` gives
    the output, `backward(dy)` the gradient of x, and `distil` makes a whole pass of learning from a teacher.  With
    products="e4m3_128" weights that are set otherwise than by `init` and `descend` need `refresh`.

    All calls but `init` may be captured in a HIP graph.  What a captured pass computes is of the weights at its replay, whether an eager
    call moved them or a replayed one.  (With products="e4m3_128" a captured step puts them into 8 bits behind itself, and a pass that is
    captured while they have moved since the last eager one also in front of itself: `refresh` before the capture saves that.)"""

    def __init__(self, depth: int, width: int, hidden: int, rows: int, dtype="bf16", act: str = "gelu",
                 checkpoints="storage", device: str = "cuda:0", norm: str = "rms", products: str = "storage", classes=None,
                 passes: str = "both"):
        import torch
        if depth < 1:
            raise LfError(LF_EINVAL, f"{depth} blocks")
        self.torch, self.depth, self.rows, self.classes = torch, depth, rows, classes
        self.dtype, _, dt = _storage(dtype)
        if checkpoints not in ("e4m3", "storage") and _storage(checkpoints)[0] != self.dtype:
            raise LfError(LF_EINVAL, f"checkpoints = {checkpoints!r}: e4m3, storage or the storage type's name")
        for name, value, allowed in (("norm", norm, ("rms", "layer")), ("products", products, ("storage", "e4m3_128")),
                                     ("passes", passes, ("both", "forward"))):
            if value not in allowed:
                raise LfError(LF_EINVAL, f"{name} = {value!r}: {' or '.join(allowed)}")
        if classes is not None and classes < 1:
            raise LfError(LF_EINVAL, f"{classes} classes")
        kept = "e4m3" if checkpoints == "e4m3" else self.dtype
        self._blocks, self._layer, self._both = products == "e4m3_128", norm == "layer", passes == "both"
        new = dict(dtype=self.dtype, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        # what the next block overwrites: the running sum, a branch, the gradients on their way down
        self._s, self._branch = (torch.empty((rows, width), **new) for _ in range(2))
        self._ds = self._du = self._dh = "none"
        if self._both:
            self._ds, self._du, self._dh = (torch.empty((rows, n), **new) for n in (width, hidden, width))
        sizes = ((hidden, width), (width, hidden), *([(classes, width)] if classes else []))
        needs = ((lf_block_linear_workspace_bytes, lf_block_linear_backward_workspace_bytes) if self._blocks
                 else (lf_linear_workspace_bytes, lf_linear_backward_workspace_bytes))
        scratch = torch.empty(max(f(rows, o, i, *(() if self._blocks else (dt,))) for f in needs for o, i in sizes), dtype=torch.uint8, device=device)
        self.out = torch.empty((rows, classes or width), **new)
        self.norms, self.ups, self.downs, self._sums = [], [], [], []
        self.w1, self.b1, self.w2, self.b2 = [], [], [], []
        make = dict(workspace=scratch, passes=passes, device=device)
        product = BlockLinear if self._blocks else Linear
        # h and u: kept as they are; with blocks of 128 the product keeps their transposed codes, and what was put in is free again,
        # or, where there is nothing to keep, the norm and the product write the next one's operand themselves
        if self._both and not self._blocks:
            h = u = kept
        elif self._both:
            h, u = torch.empty((rows, width), **new), torch.empty((rows, hidden), **new)
        else:
            def free_again(cols, kind):
                if kind == "e4m3":
                    return E4M3Matrix(rows, cols, device)
                return E4M3Blocks(rows, cols, device=device) if kind == "e4m3_128" else torch.empty((rows, cols), **new)
            h = free_again(width, kept if not self._blocks else "e4m3_128" if self._layer else self.dtype)
            u = free_again(hidden, "e4m3_128" if self._blocks else kept)
        z = "none" if act == "none" or not self._both else "e4m3_128" if self._blocks and kept == "e4m3" else kept
        for b in range(depth + (classes is not None)):
            # the running sum is updated in place; its checkpoint, or in the storage type the sum itself, is the block's
            self._sums.append(E4M3Matrix(rows, width, device) if kept == "e4m3" and self._both else torch.empty((rows, width), **new)
                              if self._both else self._s)
            self.norms.append((LayerNorm if self._layer else RmsNorm)(
                rows, width, dtype, out=h, sum=self._s if isinstance(self._sums[b], E4M3Matrix) else self._sums[b],
                dx=self._ds if self._both else None, passes=passes, device=device))
            if b == depth:
                self.head = product(rows, classes, width, dtype, y=self.out, dx=self._dh if self._both else None, **make)
                self.w_out, self.b_out = torch.empty((classes, width), **new), torch.zeros(classes, **f32)
                break
            last = b == depth - 1 and classes is None
            self.ups.append(product(rows, hidden, width, dtype, act=act, y=u, z=z, dx=self._dh if self._both else None, **make))
            self.downs.append(product(rows, width, hidden, dtype, y=self.out if last else self._branch,
                                      dx=self._du if self._both else None, **make))
            self.w1.append(torch.empty((hidden, width), **new))
            self.b1.append(torch.zeros(hidden, **f32))
            self.w2.append(torch.empty((width, hidden), **new))
            self.b2.append(torch.zeros(width, **f32))
        self._products = [*zip(self.ups, self.w1, self.b1), *zip(self.downs, self.w2, self.b2)]
        if classes is not None:
            self._products.append((self.head, self.w_out, self.b_out))
        for p, w, bias in self._products:
            (p._register if self._blocks else p.set_params)(w, bias)
        # of the weights in 8 bits: the next pass has to make them; a captured pass that does not make them reads them
        self._stale, self._relied = self._blocks, False
        self._masters = self._loss = None
        # whether a replay has filled the weights' fp32 copies, where a captured step was the first (None: no such step)
        self._filled, self._unfilled = None, torch.zeros((), dtype=torch.bool, device=device)
        self.gain = [n.gain for n in self.norms]
        self.shift = [n.shift for n in self.norms] if self._layer else []
        if self._both:
            self.dgain = [n.dgain for n in self.norms]
            self.dshift = [n.dshift for n in self.norms] if self._layer else []
            self.dw1, self.db1 = [p.dw for p in self.ups], [p.db for p in self.ups]
            self.dw2, self.db2 = [p.dw for p in self.downs], [p.db for p in self.downs]
            if classes is not None:
                self.dw_out, self.db_out = self.head.dw, self.head.db

    def init(self, seed: int = 0) -> None:
        """Random weights: variance 1 / fan-in, the second product's divided by the depth, so that the sum grows little."""
        g = self.torch.Generator(device=self.w1[0].device)
        g.manual_seed(seed)
        pairs = [(w, scale) for w1, w2 in zip(self.w1, self.w2) for w, scale in ((w1, 1.0), (w2, self.depth ** -0.5))]
        for w, scale in pairs + ([(self.w_out, 1.0)] if self.classes else []):
            v = self.torch.randn(w.shape, generator=g, device=w.device)
            w.copy_(v * (scale * w.shape[1] ** -0.5))
        self._moved()

    def refresh(self) -> None:
        """Keeps the weights as they are now in 8 bits, if the products take them so."""
        if not self._blocks:
            return
        for p, _, _ in self._products:
            p.refresh()
        if not self._capturing():              # (what is captured has not run)
            self._stale = False

    def _moved(self) -> None:
        """The weights are others now.  No replay comes back to this class to ask whether they are: a captured step makes them in 8 bits
        again, and an eager one does for the captured passes that do not."""
        if not self._blocks:
            return
        capturing = self._capturing()
        if capturing or self._relied:
            self.refresh()
        if not capturing:
            self._stale = True                 # (made by the next eager pass, of what the caller sets until then, too)

    def forward(self, x):
        if self._stale:
            self.refresh()
        elif self._blocks and not self._relied:
            self._relied = self._capturing()
        s, branch = x, None
        for b in range(self.depth):
            s, h = self._normed(b, s, branch)
            u = self.ups[b].forward(h)
            branch = self.downs[b].forward(u, residual=s if b == self.depth - 1 and self.classes is None else None)
        if self.classes is None:
            return branch
        return self.head.forward(self._normed(self.depth, s, branch)[1])

    def _normed(self, b, s, branch):
        """(the running sum, its norm) at the beginning of block b"""
        h = self.norms[b].forward(s, branch)
        s = self.norms[b].sum
        if isinstance(self._sums[b], E4M3Matrix):
            self._sums[b].first(s.shape[0]).save(s)
        return s, h

    def backward(self, dy):
        ds = dy
        if self.classes is not None:
            ds = self._norm_back(self.depth, self._product_back(self.head, dy, self.norms[self.depth].y), None)
        for b in reversed(range(self.depth)):
            du = self._product_back(self.downs[b], ds, self.ups[b].y)
            ds = self._norm_back(b, self._product_back(self.ups[b], du, self.norms[b].y), ds)
        return ds

    def _product_back(self, p, dy, x):
        return p.backward(dy) if self._blocks else p.backward(dy, x)

    def _norm_back(self, b, dh, ds):
        n, kept = dh.shape[0], self._sums[b]
        return self.norms[b].backward(dh, ds, stored=kept.first(n) if isinstance(kept, E4M3Matrix) else kept[:n])

    def distil(self, x, top_logits, top_classes, temperature: float = 1.0, weight=None):
        """A forward and a backward pass that learns from a teacher's top logits ([rows][top], f32 or bf16) of the classes that top_classes
        names (int32, negative: no entry): the loss of each row, f32, as `Distillation` has it.  The parameters' gradients are those
        of the sum of the rows' losses, each times its weight ([rows] f32, None: ones).  The logits are overwritten; the losses are a
        tensor of their own."""
        if self.classes is None or not self._both:
            raise LfError(LF_EINVAL, "distil: the net was made without classes or without its backward pass")
        if top_logits.dim() != 2:
            raise LfError(LF_EINVAL, f"top_logits: a matrix is needed, got {list(top_logits.shape)}")
        top = int(top_logits.shape[1])
        if self._loss is None:
            self._loss = Distillation(self.rows, self.classes, top, self.dtype, dlogits=self.out, device=self.w_out.device)
        # (one for every temperature and number of entries)
        loss = self._loss
        loss.top, loss.temperature, loss._loss = top, float(temperature), self.torch.empty_like(loss._loss)
        rows = loss.forward(self.forward(x), top_logits, top_classes, weight)
        self.backward(loss.dlogits)
        return rows

    def _capturing(self) -> bool:
        """Whether what is enqueued now goes into a HIP graph."""
        cuda, device = self.torch.cuda, self.w1[0].device
        if device.type != "cuda":
            return False
        if cuda.current_device() == device.index:
            return cuda.is_current_stream_capturing()
        with cuda.device(device):
            return cuda.is_current_stream_capturing()

    def descend(self, eta: float) -> None:
        """A plain gradient-descent step: every parameter less eta times its gradient.  Weights in bf16 descend in fp32 copies, made
        in the first step, and are these copies' roundings, so that steps smaller than half of bf16's add up.  A weight that was
        set to something else meanwhile goes on from there.  A step may be captured, the first among them."""
        if not self._both:
            raise LfError(LF_EINVAL, "descend: the net was made without its backward pass")
        torch = self.torch
        own = [*self.w1, *self.w2, *([self.w_out] if self.classes else [])]
        grads = [*self.dw1, *self.dw2, *([self.dw_out] if self.classes else [])]
        if self.dtype == torch.float32:
            weights = own
        else:
            if self._masters is None and self._capturing():
                # (a copy that is captured would be made again in every replay: these are filled by the first)
                self._masters, self._filled = [torch.empty_like(w, dtype=torch.float32) for w in own], self._unfilled
            elif self._masters is None:
                self._masters = [w.float() for w in own]
            weights = self._masters
            for w, master in zip(own, weights):
                same = master.to(w.dtype) == w
                if self._filled is not None:
                    same &= self._filled
                master.copy_(torch.where(same, master, w.float()))
        vectors = [*self.b1, *self.b2, *self.gain, *self.shift, *([self.b_out] if self.classes else [])]
        vector_grads = [*self.db1, *self.db2, *self.dgain, *self.dshift, *([self.db_out] if self.classes else [])]
        for p, g in zip((*weights, *vectors), (*grads, *vector_grads)):
            p.add_(g, alpha=-eta)
        for w, master in zip(own, weights):
            if master is not w:
                w.copy_(master)
        if self._filled is not None:
            self._filled.fill_(True)
        self._moved()
