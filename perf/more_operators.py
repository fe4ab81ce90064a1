"""Measured cases of the operators of a block of rows: linear layers, the norms around a block, and the update of its weights.

A case is one call on `rows` rows (images, tokens, or the pixels of a channel-innermost tensor), or on a batch of matrices:

* `kind` "linear_fwd": out = act(x w^T + bias) (+ residual), and the sum before the activation where `pre` asks for it;
* `kind` "linear_bwd": its gradients in x, w and bias from the gradient of out and the saved sum;
* `kind` "residual_norm_fwd": what stands between two blocks: r_out = r + scale * gate * norm(h), and y, the norm of that sum before it
  is rounded.  `post`: h is normed; `rms`: both norms divide by the root of the mean square alone; `gate_rows` rows share a row of gates (0: no gate),
  `sigmoid`: the gates are the sigmoids of what is given; `scale`: a factor for each channel;
* `kind` "residual_norm_bwd": its gradients in r, h, the gates, and every vector;
* `kind` "orthogonalize": `steps` Newton-Schulz steps X <- a X + (b X X^T + c (X X^T)^2) X on each of `batch` matrices.

`type` is the type of the float tensors (f32, f16, bf16); affine weights, biases, scales and statistics are f32.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_EPS = 1e-5
_STEP = (3.4445, -4.7750, 2.0315)  # coefficients of a Newton-Schulz step
_NORM_EPS = 1e-7                   # added to the norm of a matrix

# What the largest listed cases move and multiply; drawn ones stay below.
_MOST_ROWS = 1 << 26        # elements of a tensor between two blocks
_MOST_MACS = 1 << 38        # products of a linear layer
_MOST_OUT = 1 << 27         # elements of what a linear layer gives
_MOST_UPDATE = 20 << 36     # products of an update in its plain form


def _linear(name, kind, rows, cols, outs, type, act="none", residual=False, pre=False):
    return {"name": name, "kind": kind, "rows": rows, "cols": cols, "outs": outs, "type": type, "act": act, "residual": residual, "pre": pre}


def _norm(name, kind, rows, cols, type, post=True, rms=False, gate_rows=0, sigmoid=False, scale=True):
    return {"name": name, "kind": kind, "rows": rows, "cols": cols, "type": type, "post": post, "rms": rms, "gate_rows": gate_rows,
            "sigmoid": sigmoid, "scale": scale}


def _update(name, batch, rows, cols, type, steps=5):
    return {"name": name, "kind": "orthogonalize", "batch": batch, "rows": rows, "cols": cols, "type": type, "steps": steps}


def listed():
    return [
        # a 4096 -> 4096 layer for one image, as serving answers it: the weights are read once
        _linear("linear_fwd_t1_k4096_n4096_f16", "linear_fwd", 1, 4096, 4096, "f16", "relu"),
        # sizes and row lengths that fit no tile and no vector, everything in the epilogue
        _linear("linear_fwd_t777_k1001_n1283_bf16", "linear_fwd", 777, 1001, 1283, "bf16", "silu", True, True),
        # the pixels of a 13x13 stage of 20 images, widened fourfold, in fp32
        _linear("linear_fwd_t3380_k384_n1536_f32", "linear_fwd", 20 * 13 * 13, 384, 1536, "f32", "gelu"),
        # a training batch through a wide layer that keeps what its gradient needs: the largest product
        _linear("linear_fwd_t8192_k4096_n8192_bf16", "linear_fwd", 8192, 4096, 8192, "bf16", "gelu", False, True),
        # the gradients of a training head over a large vocabulary of odd size
        _linear("linear_bwd_t2048_k1024_n50257_bf16", "linear_bwd", 2048, 1024, 50257, "bf16"),
        # every pixel of a 56x56 stage of 64 images: a very long sum for few weights
        _linear("linear_bwd_t200704_k192_n768_f16", "linear_bwd", 64 * 56 * 56, 192, 768, "f16", "gelu"),
        # between two blocks for one image: launch and host cost
        _norm("residual_norm_fwd_t1_d4096_f16", "residual_norm_fwd", 1, 4096, "f16", rms=True),
        # the pixels of a 14x14 stage of 256 images, gates for each image's channels
        _norm("residual_norm_fwd_t50176_d768_bf16", "residual_norm_fwd", 256 * 14 * 14, 768, "bf16", gate_rows=196, sigmoid=True),
        # the gradients at a 13x13 stage of 20 images, no norm behind the block, gates for each image's channels
        _norm("residual_norm_bwd_t3380_d384_f32", "residual_norm_bwd", 20 * 13 * 13, 384, "f32", post=False, gate_rows=169),
        # the gradients of a training batch of wide rows with gates of their own: the largest tensor
        _norm("residual_norm_bwd_t16384_d4096_bf16", "residual_norm_bwd", 16384, 4096, "bf16", rms=True, gate_rows=1, scale=False),
        # the layers of a narrow stage, updated together
        _update("orthogonalize_b24_192x768_f32", 24, 192, 768, "f32"),
        # one wide square layer: the largest update
        _update("orthogonalize_b1_4096x4096_bf16", 1, 4096, 4096, "bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; two of three are multiples of what vectors hold."""
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))
    return max(lo, n // 16 * 16) if n >= 64 and rng.random() < 0.6 else n


def draw(rng):
    kind = rng.choice(("linear_fwd", "linear_fwd", "linear_bwd", "residual_norm_fwd", "residual_norm_bwd", "orthogonalize"))
    type = rng.choice(("f32", "f16", "bf16"))
    if kind in ("linear_fwd", "linear_bwd"):
        cols, outs = _log(rng, 16, 16384), _log(rng, 10, 65536)
        most = _MOST_MACS // (8 if type == "f32" else 1) // (2 if kind == "linear_bwd" else 1)
        rows = _log(rng, 1, max(1, min(262144, most // (cols * outs), _MOST_OUT // outs, _MOST_OUT // cols)))
        return {"kind": kind, "rows": rows, "cols": cols, "outs": outs, "type": type, "act": rng.choice(("none", "relu", "gelu", "silu")),
                "residual": kind == "linear_fwd" and rng.random() < 0.5, "pre": kind == "linear_fwd" and rng.random() < 0.3}
    if kind in ("residual_norm_fwd", "residual_norm_bwd"):
        cols = _log(rng, 16, 16384)
        rows = _log(rng, 1, min(262144, _MOST_ROWS // cols))
        return {"kind": kind, "rows": rows, "cols": cols, "type": type, "post": rng.random() < 0.6, "rms": rng.random() < 0.5,
                "gate_rows": rng.choice((0, 1, 49, 196)), "sigmoid": rng.random() < 0.5, "scale": rng.random() < 0.6}
    steps = rng.choice((4, 5, 5, 6))
    rows, cols = _log(rng, 16, 4096), _log(rng, 16, 4096)
    small, large = min(rows, cols), max(rows, cols)
    each = steps * small * small * (2 * large + small) * (4 if type == "f32" else 1)
    return {"kind": kind, "batch": _log(rng, 1, max(1, min(64, _MOST_UPDATE // each))), "rows": rows, "cols": cols, "type": type, "steps": steps}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, kind, f32 = _TORCH[case["type"]], case["kind"], torch.float32
    rows, cols = case["rows"], case["cols"]

    def normal(*shape, sigma=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(sigma).add_(mean)

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s = {"case": case}
    if kind == "orthogonalize":
        # a layer's gradient: some strong directions above a floor of weak ones, of any size
        batch = case["batch"]
        strong = max(1, min(rows, cols) // 8)
        x = torch.matmul(normal(batch, rows, strong), normal(batch, strong, cols)).mul_(strong ** -0.5)
        s["x"] = x.add_(normal(batch, rows, cols, sigma=0.3)).mul_(normal(batch, 1, 1).abs_().add_(0.1).mul_(1e-3)).to(dt)
        s["out"] = empty(batch, rows, cols)
        return s
    if kind in ("linear_fwd", "linear_bwd"):
        outs = case["outs"]
        s["x"] = normal(rows, cols).mul_(normal(rows, 1).abs_().add_(0.5)).to(dt)
        s["w"] = normal(outs, cols, sigma=cols ** -0.5).to(dt)
        s["bias"] = normal(outs, sigma=0.1)
        if kind == "linear_fwd":
            s["residual"] = normal(rows, outs).to(dt) if case["residual"] else None
            s["pre"] = empty(rows, outs) if case["pre"] else None
            s["out"] = empty(rows, outs)
        else:
            # the saved sum has the distribution that the forward pass leaves
            s["pre"] = normal(rows, outs).mul_(normal(rows, 1).abs_().add_(0.5)).to(dt) if case["act"] != "none" else None
            s["dout"] = normal(rows, outs, sigma=0.1).to(dt)
            s.update(dx=empty(rows, cols), dw=empty(outs, cols), dbias=empty(outs, dtype=f32))
        return s
    s["r"] = normal(rows, cols).mul_(normal(rows, 1).abs_().add_(0.5)).add_(normal(rows, 1, sigma=0.5)).to(dt)
    s["h"] = normal(rows, cols, sigma=0.5).mul_(normal(rows, 1).abs_().add_(0.5)).add_(normal(rows, 1, sigma=0.2)).to(dt)
    s["gate"] = normal(-(-rows // case["gate_rows"]), cols, sigma=0.7, mean=0.5).to(dt) if case["gate_rows"] else None
    s["gamma_h"], s["beta_h"] = (normal(cols, sigma=0.2, mean=1.0), normal(cols, sigma=0.2)) if case["post"] else (None, None)
    s["scale"] = normal(cols, sigma=0.1, mean=0.5) if case["scale"] else None
    s["gamma"], s["beta"] = normal(cols, sigma=0.2, mean=1.0), normal(cols, sigma=0.2)
    if kind == "residual_norm_fwd":
        s.update(r_out=empty(rows, cols), y=empty(rows, cols), stats=empty(rows, 4, dtype=f32))
        return s
    # what the forward pass left behind, and the gradients that reach its outputs
    s["r_out"], _, s["stats"] = _plain_norm(s)
    del s["r"]
    s["dr_out"], s["dy"] = normal(rows, cols, sigma=0.1).to(dt), normal(rows, cols, sigma=0.1).to(dt)
    s.update(dr=empty(rows, cols), dh=empty(rows, cols), dgate=empty(*s["gate"].shape) if case["gate_rows"] else None)
    for k in ("gamma_h", "beta_h", "scale", "gamma", "beta"):
        s["d" + k] = empty(cols, dtype=f32) if s[k] is not None else None
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.5 ** 0.5))
    return z * torch.sigmoid(z) if act == "silu" else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    p = torch.sigmoid(z)
    return p * (1.0 + z * (1.0 - p))


def _plain_linear(s):
    dt, act = s["x"].dtype, s["case"]["act"]
    z = s["x"].float() @ s["w"].float().t() + s["bias"]
    out = _act(z, act)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return (out.to(dt), z.to(dt)) if s["case"]["pre"] else (out.to(dt),)


def _plain_linear_bwd(s):
    dt, act = s["x"].dtype, s["case"]["act"]
    dz = s["dout"].float()
    if act != "none":
        dz = dz * _act_slope(s["pre"].float(), act)
    return (dz @ s["w"].float()).to(dt), (dz.t() @ s["x"].float()).to(dt), dz.sum(0)


def _stats(x, rms):
    mean = torch.zeros_like(x[:, :1]) if rms else x.mean(1, keepdim=True)
    return mean, torch.rsqrt((x - mean).square().mean(1, keepdim=True) + _EPS)


def _gates(s, gate, rows):
    """The gates as they multiply, a row of them for each row."""
    g = torch.sigmoid(gate) if s["case"]["sigmoid"] else gate
    return g[torch.arange(rows, device=g.device) // s["case"]["gate_rows"]]


def _plain_norm(s):
    c, r, u = s["case"], s["r"].float(), s["h"].float()
    mean_h, rstd_h = torch.zeros_like(r[:, :1]), torch.ones_like(r[:, :1])
    if c["post"]:
        mean_h, rstd_h = _stats(u, c["rms"])
        u = (u - mean_h) * rstd_h * s["gamma_h"] + s["beta_h"]
    if c["gate_rows"]:
        u = u * _gates(s, s["gate"].float(), c["rows"])
    if c["scale"]:
        u = u * s["scale"]
    x = r + u
    mean, rstd = _stats(x, c["rms"])
    y = (x - mean) * rstd * s["gamma"] + s["beta"]
    return x.to(s["r"].dtype), y.to(s["r"].dtype), torch.cat((mean_h, rstd_h, mean, rstd), 1)


def _norm_slope(g, xh, rstd, rms):
    """The gradient in a row from the gradient g of the normed row xh."""
    along = xh * (g * xh).mean(1, keepdim=True)
    return rstd * (g - along) if rms else rstd * (g - g.mean(1, keepdim=True) - along)


def _plain_norm_bwd(s):
    c, dt = s["case"], s["h"].dtype
    mean_h, rstd_h, mean, rstd = s["stats"].split(1, 1)
    dy, xh = s["dy"].float(), (s["r_out"].float() - mean) * rstd
    dr = s["dr_out"].float() + _norm_slope(dy * s["gamma"], xh, rstd, c["rms"])
    hh = (s["h"].float() - mean_h) * rstd_h
    u = hh * s["gamma_h"] + s["beta_h"] if c["post"] else hh
    p, out = dr, [dr.to(dt)]
    if c["gate_rows"]:
        gate = s["gate"].float()
        q = dr * u * s["scale"] if c["scale"] else dr * u
        if c["gate_rows"] == 1:
            dgate = q
        else:
            dgate = torch.zeros_like(gate).index_add_(0, torch.arange(c["rows"], device=q.device) // c["gate_rows"], q)
        if c["sigmoid"]:
            dgate = dgate * torch.sigmoid(gate) * (1.0 - torch.sigmoid(gate))
        p = dr * _gates(s, gate, c["rows"])
    du = p * s["scale"] if c["scale"] else p
    out.append((_norm_slope(du * s["gamma_h"], hh, rstd_h, c["rms"]) if c["post"] else du).to(dt))
    if c["gate_rows"]:
        out.append(dgate.to(dt))
    if c["post"]:
        out += [(du * hh).sum(0), du.sum(0)]
    if c["scale"]:
        out.append((p * u).sum(0))
    return (*out, (dy * xh).sum(0), dy.sum(0))


def _plain_update(s):
    x = s["x"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    a, b, c = _STEP
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + _NORM_EPS)
    for _ in range(s["case"]["steps"]):
        m = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * m + c * torch.matmul(m, m), x)
    return (x.transpose(1, 2) if tall else x).to(s["x"].dtype)


def _plain(s):
    kind = s["case"]["kind"]
    return {"linear_fwd": _plain_linear, "linear_bwd": _plain_linear_bwd, "residual_norm_fwd": _plain_norm, "residual_norm_bwd": _plain_norm_bwd,
            "orthogonalize": _plain_update}[kind](s)


# ---- the framework's operators ---------------------------------------------------------------------------------------


def _plan(s):
    """The descriptor and the workspace that a program makes once for its sizes and keeps."""
    from paper_1611_06945_amd import binding as B

    c = s["case"]
    kind, rows, cols = c["kind"], c["rows"], c["cols"]
    dt = {"f32": B.CONV_F32, "f16": B.CONV_F16, "bf16": B.CONV_BF16}[c["type"]]
    need = 0
    if kind in ("linear_fwd", "linear_bwd"):
        s["desc"] = B.make_linear_desc(rows, c["outs"], cols, dt, act=c["act"])
        need = B.linear_workspace_bytes(s["desc"]) if kind == "linear_fwd" else B.linear_bwd_workspace_bytes(s["desc"])
    elif kind == "orthogonalize":
        s["desc"] = B.make_orthogonal_desc(rows, cols, dt, batch=c["batch"], steps=c["steps"], coefficients=_STEP, eps=_NORM_EPS)
        need = B.orthogonalize_workspace_bytes(s["desc"])
    else:
        s["desc"] = B.make_residual_norm_desc(rows, cols, dt, eps=_EPS, rms=c["rms"], post=c["post"], gate_rows=c["gate_rows"], sigmoid=c["sigmoid"])
        need = B.residual_norm_bwd_workspace_bytes(s["desc"]) if kind == "residual_norm_bwd" else 0
    s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    s["B"] = B


def _own(s):
    if "B" not in s:
        _plan(s)
    B, kind, ws = s["B"], s["case"]["kind"], s["ws"]
    if kind == "linear_fwd":
        B.linear_fwd(s["desc"], s["x"], s["w"], s["bias"], s["residual"], s["out"], s["pre"], ws, ws.numel())
        return (s["out"], s["pre"]) if s["case"]["pre"] else (s["out"],)
    if kind == "linear_bwd":
        B.linear_bwd(s["desc"], s["x"], s["w"], s["pre"], s["dout"], s["dx"], s["dw"], s["dbias"], ws, ws.numel())
        return s["dx"], s["dw"], s["dbias"]
    if kind == "orthogonalize":
        B.orthogonalize(s["desc"], s["x"], s["out"], ws, ws.numel())
        return s["out"]
    if kind == "residual_norm_fwd":
        B.residual_norm_fwd(s["desc"], s["r"], s["h"], s["gate"], s["gamma_h"], s["beta_h"], s["scale"], s["gamma"], s["beta"], s["r_out"], s["y"], s["stats"])
        return s["r_out"], s["y"], s["stats"]
    B.residual_norm_bwd(s["desc"], s["r_out"], s["h"], s["gate"], s["gamma_h"], s["beta_h"], s["scale"], s["gamma"], s["stats"], s["dr_out"], s["dy"],
                        s["dr"], s["dh"], s["dgate"], s["dgamma_h"], s["dbeta_h"], s["dscale"], s["dgamma"], s["dbeta"], ws, ws.numel())
    return tuple(s[k] for k in ("dr", "dh", "dgate", "dgamma_h", "dbeta_h", "dscale", "dgamma", "dbeta") if s[k] is not None)


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    t, d, es, kind = case["rows"], case["cols"], _BYTES[case["type"]], case["kind"]
    if kind == "linear_fwd":
        n = case["outs"]
        return {"bytes": (t * d + n * d + t * n * (1 + case["residual"] + case["pre"])) * es + 4 * n, "flops": 2 * t * d * n}
    if kind == "linear_bwd":
        n = case["outs"]
        return {"bytes": (2 * t * d + 2 * n * d + t * n * (1 if case["act"] == "none" else 2)) * es + 4 * n, "flops": 4 * t * d * n}
    if kind == "orthogonalize":
        # X X^T and its square are symmetric: half of each
        small, large, batch = min(t, d), max(t, d), case["batch"]
        return {"bytes": 2 * batch * t * d * es, "flops": batch * case["steps"] * small * small * (3 * large + small)}
    gates = -(-t // case["gate_rows"]) * d * es if case["gate_rows"] else 0
    vectors = 2 + 2 * case["post"] + case["scale"]
    if kind == "residual_norm_fwd":
        return {"bytes": 4 * t * d * es + gates + 4 * d * vectors + 16 * t, "flops": (18 + 8 * case["post"]) * t * d}
    return {"bytes": 6 * t * d * es + 2 * gates + 8 * d * vectors + 16 * t, "flops": (22 + 12 * case["post"]) * t * d}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------


def _exact_act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _exact_norm(x, rms):
    mean = 0.0 * x.sum(1) if rms else x.sum(1) / x.shape[1]
    x = x - mean[:, None]
    rstd = ((x * x).sum(1) / x.shape[1] + _EPS) ** -0.5
    return x * rstd[:, None], mean, rstd


def _exact_branch(c, r, h, gate, gamma_h, beta_h, scale):
    """r + scale * gate * norm(h), and the statistics of h."""
    u, mean, rstd = _exact_norm(h, c["rms"]) if c["post"] else (h, 0.0 * h[:, 0], 1.0 + 0.0 * h[:, 0])
    if c["post"]:
        u = gamma_h * u + beta_h
    if c["gate_rows"]:
        each = gate.repeat_interleave(c["gate_rows"], 0)[: c["rows"]]
        u = u / (1.0 + torch.exp(-each)) if c["sigmoid"] else u * each
    return r + (u * scale if c["scale"] else u), mean, rstd


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "orthogonalize":
        x = s["x"].double()
        a, b, c = _STEP
        x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + _NORM_EPS)
        for _ in range(case["steps"]):
            # on the right, from X^T X: the same polynomial of X
            m = torch.matmul(x.transpose(1, 2).contiguous(), x) if case["rows"] >= case["cols"] else None
            if m is not None:
                x = a * x + torch.matmul(x, b * m + c * torch.matmul(m, m))
            else:
                y = torch.matmul(torch.matmul(x, x.transpose(1, 2).contiguous()), x)
                x = a * x + b * y + c * torch.matmul(torch.matmul(x, x.transpose(1, 2).contiguous()), y)
        return x
    if kind == "linear_fwd":
        z = torch.addmm(s["bias"].double(), s["x"].double(), s["w"].double().t())
        out = _exact_act(z, case["act"])
        out = out + s["residual"].double() if case["residual"] else out
        return (out, z) if case["pre"] else (out,)
    if kind == "linear_bwd":
        dz = s["dout"].double()
        if case["act"] != "none":
            z = s["pre"].double().requires_grad_()
            (dz,) = torch.autograd.grad(_exact_act(z, case["act"]), z, dz)
        return torch.mm(dz, s["w"].double()), torch.mm(s["x"].double().t(), dz).t(), torch.mv(dz.t(), torch.ones_like(dz[:, 0]))
    gate, gamma_h, beta_h, scale = (None if s[k] is None else s[k].double() for k in ("gate", "gamma_h", "beta_h", "scale"))
    if kind == "residual_norm_fwd":
        r_out, mean_h, rstd_h = _exact_branch(case, s["r"].double(), s["h"].double(), gate, gamma_h, beta_h, scale)
        y, mean, rstd = _exact_norm(r_out, case["rms"])
        return r_out, s["gamma"].double() * y + s["beta"].double(), torch.stack((mean_h, rstd_h, mean, rstd), 1)
    # the saved statistics are inputs: the norms' gradients by their parts along the row of ones and along the normed row
    def through(x, mean, rstd, g):
        xh = (x.double() - mean[:, None]) * rstd[:, None]
        ones = torch.ones_like(xh[0])
        along_xh = torch.linalg.vecdot(g, xh) / xh.shape[1]
        along_ones = 0.0 * along_xh if case["rms"] else torch.mv(g, ones) / xh.shape[1]
        return (g - torch.outer(along_ones, ones) - along_xh[:, None] * xh) * rstd[:, None], xh

    mean_h, rstd_h, mean, rstd = s["stats"].double().unbind(1)
    dy = s["dy"].double()
    dx, xh = through(s["r_out"], mean, rstd, dy * s["gamma"].double())
    dr, dgamma, dbeta = s["dr_out"].double() + dx, (dy * xh).sum(0), dy.sum(0)
    del dx, dy, xh
    # ... and through the sum by differentiation
    hh = ((s["h"].double() - mean_h[:, None]) * rstd_h[:, None]).requires_grad_()
    leaves = [t.requires_grad_() for t in (gate, gamma_h, beta_h, scale) if t is not None]
    plain = dict(case, post=False)
    u = gamma_h * hh + beta_h if case["post"] else hh
    du, *rest = torch.autograd.grad(_exact_branch(plain, torch.zeros_like(dr), u, gate, None, None, scale)[0], [hh, *leaves], dr)
    return (dr, through(s["h"], mean_h, rstd_h, du)[0] if case["post"] else du, *rest, dgamma, dbeta)
