"""Blocks of rows between the convolutions' features and the head, on the operators of the C ABI, and the update of their weights.

    y = norm(r);   h = act(y w1^T + b1) w2^T + b2;   r <- r + scale * gate * norm(h);   y = norm(r)  for the next block

`TrainingBlock` is one such block with its gradients: two linear layers, and one call for all that stands between two blocks (the norm
behind the layers, the gate, the residual sum and the norm before the next block).  Blocks of one width are chained by handing on (r, y), and
their gradients back by (dr, dy); the head's features are the last block's r.

`OrthogonalUpdate` turns the gradients of weights of one shape into directions with singular values near one (momentum, then Newton-Schulz steps).

    python -m paper_1611_06945_amd.block           # trains two blocks and a head on synthetic features
"""
from __future__ import annotations

from . import binding as B
from .head import GPU, TrainingHead, _check, _code

WEIGHTS = ("w1", "w2")
VECTORS = ("b1", "b2", "gamma_h", "beta_h", "scale", "gamma", "beta")


def _current(torch, device):
    """Kernels are launched on the current device."""
    if device.type == "cuda" and torch.cuda.current_device() != device.index:
        raise ValueError("the buffers are on %s, the current device is %d" % (device, torch.cuda.current_device()))


class TrainingBlock:
    def __init__(self, rows: int, D: int, hidden: int, dtype, act: str = "gelu", rms: bool = False, post: bool = True, gate_rows: int = 0,
                 sigmoid: bool = False, last: bool = False, eps: float = 1e-5, device="cuda"):
        """Buffers and descriptors for batches of `rows` rows [rows][D] in `dtype`.  rms, post, gate_rows, sigmoid: as in make_residual_norm_desc;
        last: there is no norm behind the sum (y is None, and no gamma and beta)."""
        import torch

        if torch.device(device).type != GPU:
            raise ValueError("a block on %s: its kernels run on the GPU" % device)
        self.torch, self.rows, self.D, self.hidden, self.dtype, self.gate_rows, self.last = torch, rows, D, hidden, dtype, gate_rows, last
        code = _code(torch, dtype)
        new = lambda *shape: torch.empty(*shape, dtype=dtype, device=device)  # noqa: E731
        vec = lambda *shape: torch.empty(*shape, dtype=torch.float32, device=device)  # noqa: E731
        self.shapes = {"w1": (hidden, D), "w2": (D, hidden), "b1": (hidden,), "b2": (D,), "scale": (D,)}
        if post:
            self.shapes.update(gamma_h=(D,), beta_h=(D,))
        if not last:
            self.shapes.update(gamma=(D,), beta=(D,))
        gates = -(-rows // gate_rows) if gate_rows else 0
        self.pre, self.a, self.h, self.r_out, self.stats = new(rows, hidden), new(rows, hidden), new(rows, D), new(rows, D), vec(rows, 4)
        self.y = None if last else new(rows, D)
        self.da, self.dh, self.dr, self.dy = new(rows, hidden), new(rows, D), new(rows, D), new(rows, D)
        self.dgate = new(gates, D) if gate_rows else None
        self.grads = {k: new(*s) if k in WEIGHTS else vec(*s) for k, s in self.shapes.items()}
        self.first = B.make_linear_desc(rows, hidden, D, code, act=act)
        self.second = B.make_linear_desc(rows, D, hidden, code)
        self.norm = B.make_residual_norm_desc(rows, D, code, eps, rms, post, gate_rows, sigmoid)
        need = max([B.residual_norm_bwd_workspace_bytes(self.norm)] + [f(d) for d in (self.first, self.second) for f in (B.linear_workspace_bytes, B.linear_bwd_workspace_bytes)])
        self.ws = torch.empty(max(256, need), dtype=torch.uint8, device=device)
        self.saved = None

    def _rows(self, name, t):
        _check(name, t, self.dtype, (self.rows, self.D), self.h.device)

    def forward(self, r, y, weights, gate=None, stream=None):
        """r and its norm y, [rows][D] of the block's type; weights: dict of w1 [hidden][D], w2 [D][hidden] of that type and fp32 vectors b1, b2, scale and,
        where the block has their norms, gamma_h, beta_h, gamma, beta; gate: [gates][D] of the type, or None.  All dense.  -> (r_out, y_out), views of the
        block's own buffers; keeps what backward() needs."""
        dev, f32 = self.h.device, self.torch.float32
        _current(self.torch, dev)
        self._rows("r", r)
        self._rows("y", y)
        if self.rows and self.y is not None and y.data_ptr() == self.y.data_ptr():
            raise ValueError("y is the block's own result, which this pass replaces before backward() reads it")
        if set(weights) != set(self.shapes):
            raise ValueError("weights must be %s; they are %s" % (sorted(self.shapes), sorted(weights)))
        for k, s in self.shapes.items():
            _check(k, weights[k], self.dtype if k in WEIGHTS else f32, s, dev)
        if (gate is None) != (self.gate_rows == 0):
            raise ValueError("a block with gate_rows = %d and %s gate" % (self.gate_rows, "no" if gate is None else "a"))
        if gate is not None:
            _check("gate", gate, self.dtype, tuple(self.dgate.shape), dev)
        p, ws, n = weights, self.ws, self.ws.numel()
        self.saved = None
        B.linear_fwd(self.first, y, p["w1"], p["b1"], None, self.a, self.pre, ws, n, stream)
        B.linear_fwd(self.second, self.a, p["w2"], p["b2"], None, self.h, None, ws, n, stream)
        B.residual_norm_fwd(self.norm, r, self.h, gate, p.get("gamma_h"), p.get("beta_h"), p["scale"], p.get("gamma"), p.get("beta"), self.r_out, self.y, self.stats,
                            stream)
        self.saved = (y, p, gate)
        return self.r_out, self.y

    def backward(self, dr_out, dy_out=None, stream=None):
        """The gradients in r_out and in y_out (None where last, or where nothing comes from there), dense [rows][D] of the block's type -> (dr, dy), the gradients
        in r and in y; those in the weights are in self.grads, that in the gate in self.dgate.  Once for each forward(), whose inputs and whose r_out have to be as they were."""
        if self.saved is None:
            raise RuntimeError("backward() needs a forward() of its own")
        if dy_out is not None and self.last:
            raise ValueError("a last block has no y")
        _current(self.torch, self.h.device)
        self._rows("dr_out", dr_out)
        if dy_out is not None:
            self._rows("dy_out", dy_out)
        y, p, gate = self.saved
        g, ws, n = self.grads, self.ws, self.ws.numel()
        B.residual_norm_bwd(self.norm, self.r_out, self.h, gate, p.get("gamma_h"), p.get("beta_h"), p["scale"], p.get("gamma"), self.stats, dr_out, dy_out, self.dr,
                            self.dh, self.dgate, g.get("gamma_h"), g.get("beta_h"), g["scale"], g.get("gamma"), g.get("beta"), ws, n, stream)
        B.linear_bwd(self.second, self.a, p["w2"], None, self.dh, self.da, g["w2"], g["b2"], ws, n, stream)
        B.linear_bwd(self.first, y, p["w1"], self.pre, self.da, self.dy, g["w1"], g["b1"], ws, n, stream)
        self.saved = None
        return self.dr, self.dy


class OrthogonalUpdate:
    def __init__(self, count: int, rows: int, cols: int, dtype, momentum: float = 0.95, nesterov: bool = True, steps: int = 5,
                 coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7, device="cuda"):
        """For `count` weights [rows][cols]; the steps are computed on `dtype`, the momentum is kept in fp32.  fp16 is the result's type alone: gradients and their
        momentum may leave its range, so the steps are computed on fp32."""
        import torch

        if torch.device(device).type != GPU:
            raise ValueError("an update on %s: its kernels run on the GPU" % device)
        self.torch, self.momentum, self.nesterov = torch, float(momentum), bool(nesterov)
        shape = (count, rows, cols)
        self.sum = torch.zeros(*shape, dtype=torch.float32, device=device)
        self.direction = torch.empty(*shape, dtype=dtype, device=device)
        self.x = torch.empty(*shape, dtype=torch.float32, device=device) if dtype == torch.float16 else self.direction
        self.desc = B.make_orthogonal_desc(rows, cols, _code(torch, self.x.dtype), count, steps, coefficients, eps)
        self.ws = torch.empty(max(256, B.orthogonalize_workspace_bytes(self.desc)), dtype=torch.uint8, device=device)

    def step(self, grads):
        """grads: the `count` gradients [rows][cols], of any float type -> their directions [count][rows][cols], the update's own buffer.  On torch's current stream."""
        if len(grads) != self.sum.shape[0]:
            raise ValueError("%d gradients for an update of %d" % (len(grads), self.sum.shape[0]))
        for g in grads:
            if g.shape != self.sum.shape[1:] or g.device != self.sum.device or not g.is_floating_point():
                raise ValueError("a gradient must be %s of a float type on %s; it is %s %s on %s" % (
                    list(self.sum.shape[1:]), self.sum.device, g.dtype, list(g.shape), g.device))
        _current(self.torch, self.sum.device)
        self.sum.mul_(self.momentum)
        for i, g in enumerate(grads):
            self.sum[i].add_(g)
            self.x[i].copy_(self.sum[i].mul(self.momentum).add_(g) if self.nesterov else self.sum[i])
        B.orthogonalize(self.desc, self.x, self.x, self.ws, self.ws.numel())
        if self.x is not self.direction:
            self.direction.copy_(self.x)
        return self.direction


def start_weights(block, generator):
    """fp32 weights of a block to start from: random layers, ones, zeros, and a small scale."""
    torch, dev = block.torch, block.h.device
    out = {}
    for k, s in block.shapes.items():
        if k in WEIGHTS:
            out[k] = torch.randn(*s, generator=generator, device=dev) * s[1] ** -0.5
        else:
            out[k] = torch.full(s, {"gamma": 1.0, "gamma_h": 1.0, "scale": 0.1}.get(k, 0.0), device=dev)
    return out


def demo(images: int = 8, pixels: int = 49, D: int = 192, hidden: int = 768, classes: int = 100, steps: int = 30, rate: float = 0.02, log=print):
    """Trains two blocks with gates for each image, and a head, on features around one random centre a class; returns the mean log probabilities
    before and after."""
    import torch

    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rows, dt = images * pixels, torch.bfloat16
    centres = torch.randn(classes, D, generator=g, device="cuda")
    target = torch.randint(0, classes, (rows,), generator=g, device="cuda")
    r0 = (centres[target] + torch.randn(rows, D, generator=g, device="cuda")).to(dt)
    gate = torch.randn(images, D, generator=g, device="cuda").to(dt)
    y0 = torch.empty_like(r0)
    blocks = [TrainingBlock(rows, D, hidden, dt, gate_rows=pixels, sigmoid=True, last=i == 1) for i in range(2)]
    weights = [start_weights(b, g) for b in blocks]
    updates = {k: OrthogonalUpdate(len(blocks), *blocks[0].shapes[k], dtype=dt) for k in WEIGHTS}
    head, norm = TrainingHead(rows, D, classes, dt), B.make_norm_desc(rows, D, B.CONV_BF16)
    w, gamma, beta = torch.randn(classes, D, generator=g, device="cuda") * D ** -0.5, torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    g_logp = torch.full((rows,), -1.0 / rows, device="cuda")
    seen = []
    for step in range(steps):
        used = [{k: v.to(dt) if k in WEIGHTS else v for k, v in p.items()} for p in weights]
        B.layernorm_fwd(norm, r0, None, None, y0)
        r, y = r0, y0
        for b, p in zip(blocks, used):
            r, y = b.forward(r, y, p, gate)
        logp, _ = head.forward(r, gamma, beta, w.to(dt), target)
        seen.append(float(logp.mean()))
        dr, dgamma, dbeta, dw = head.backward(g_logp)
        dy = None
        for b in reversed(blocks):
            dr, dy = b.backward(dr, dy)
        for k, u in updates.items():
            moved = u.step([b.grads[k] for b in blocks])
            for p, d in zip(weights, moved):
                p[k].sub_(d.float() * rate)
        for p, b in zip(weights, blocks):
            for k in p:
                if k in VECTORS:
                    p[k].sub_(b.grads[k] * rate)
        for p, d in ((w, dw), (gamma, dgamma), (beta, dbeta)):
            p.sub_(d.float() * rate)
        if step % 10 == 0 or step == steps - 1:
            log("step %3d: mean log probability %8.4f" % (step, seen[-1]))
    return seen[0], seen[-1]


if __name__ == "__main__":
    demo()
