"""Measured cases of the operators at the end of a network: layer norm, 8-bit linear layers and log probabilities.

A case is one call, or one pair of calls that a program always makes together, on `rows` rows (images, tokens, or the
pixels of a channel-innermost tensor):

* `kind` "norm_fwd", "norm_bwd": layer norm over `cols` channels, and its gradients (dx, dgamma, dbeta);
* `kind` "linear": float rows quantised to 8 bits with a scale a row, then multiplied with 8-bit weights that carry a scale
  for each output channel;
* `kind` "norm_linear": the same behind a layer norm, whose result is written in 8 bits at once;
* `kind` "logprob_fwd": log probability of one given token a row, logsumexp, entropy, and the `top` likeliest tokens;
* `kind` "logprob_bwd": the gradient of the log probability and of the entropy in the logits.

`type` is the type of the float tensors (f32, f16, bf16); affine weights, biases, scales, statistics and log probabilities
are f32.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_EPS = 1e-5
_INF = float("inf")

# What the largest listed cases move and multiply; drawn ones stay below.
_MOST_NORM = 1 << 26    # elements of a normalised tensor
_MOST_LOGITS = 1 << 28  # elements of a tensor of logits
_MOST_MACS = 1 << 38    # products of a linear layer


def _norm(name, kind, rows, cols, type):
    return {"name": name, "kind": kind, "rows": rows, "cols": cols, "type": type}


def _linear(name, kind, rows, cols, outs, type, relu=False):
    return {"name": name, "kind": kind, "rows": rows, "cols": cols, "outs": outs, "type": type, "relu": relu}


def _logprob(name, kind, rows, cols, type, top, masked):
    return {"name": name, "kind": kind, "rows": rows, "cols": cols, "type": type, "top": top, "masked": masked}


def listed():
    return [
        # the features of one image before its classifier: the smallest call, launch and host cost
        _norm("norm_fwd_t1_d4096_f16", "norm_fwd", 1, 4096, "f16"),
        # every pixel of a 56x56 stage of 64 images, channel-innermost with 192 channels: very many short rows
        _norm("norm_fwd_t200704_d192_f32", "norm_fwd", 64 * 56 * 56, 192, "f32"),
        # the gradients at the pixels of a 13x13 stage of 20 images
        _norm("norm_bwd_t3380_d384_f16", "norm_bwd", 20 * 13 * 13, 384, "f16"),
        # ... and of a training batch of wide rows: the largest of its kind
        _norm("norm_bwd_t16384_d4096_bf16", "norm_bwd", 16384, 4096, "bf16"),
        # a 4096 -> 4096 fully connected layer for one image: the weights are read once
        _linear("linear_t1_k4096_n4096_f16", "linear", 1, 4096, 4096, "f16", True),
        # a 1000-way classifier on 20 images, fp32 features
        _linear("linear_t20_k4096_n1000_f32", "linear", 20, 4096, 1000, "f32"),
        # sizes that fit no tile, behind a layer norm
        _linear("norm_linear_t777_k1001_n1283_bf16", "norm_linear", 777, 1001, 1283, "bf16"),
        # a throughput batch through a wide layer: the largest product
        _linear("linear_t8192_k4096_n8192_bf16", "linear", 8192, 4096, 8192, "bf16"),
        # one row of a large vocabulary, as each step of serving answers it, with the likeliest alternatives
        _logprob("logprob_fwd_t1_v131072_f32", "logprob_fwd", 1, 131072, "f32", 20, False),
        # scoring a batch of tokens; a vocabulary of odd size with masked entries
        _logprob("logprob_fwd_t2048_v50257_bf16", "logprob_fwd", 2048, 50257, "bf16", 5, True),
        # a classifier's loss on a batch of images: 1000 classes
        _logprob("logprob_bwd_t1280_v1000_f32", "logprob_bwd", 1280, 1000, "f32", 0, False),
        # the gradient of a training batch over a large vocabulary: the largest tensor
        _logprob("logprob_bwd_t2048_v131072_bf16", "logprob_bwd", 2048, 131072, "bf16", 0, False),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; two of three are multiples of what vectors hold."""
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return max(lo, n // 16 * 16) if n >= 64 and rng.random() < 0.6 else n


def draw(rng):
    kind = rng.choice(("norm_fwd", "norm_bwd", "linear", "norm_linear", "logprob_fwd", "logprob_bwd"))
    type = rng.choice(("f32", "f16", "bf16"))
    if kind in ("norm_fwd", "norm_bwd"):
        cols = _log(rng, 16, 16384)
        return {"kind": kind, "rows": _log(rng, 1, min(262144, _MOST_NORM // cols)), "cols": cols, "type": type}
    if kind in ("linear", "norm_linear"):
        cols, outs = _log(rng, 32, 16384), _log(rng, 10, 32768)
        rows = _log(rng, 1, min(16384, _MOST_MACS // (cols * outs)))
        return {"kind": kind, "rows": rows, "cols": cols, "outs": outs, "relu": rng.random() < 0.5,
                "type": type if kind == "linear" else rng.choice(("f16", "bf16"))}
    cols = _log(rng, 10, 262144)
    rows = _log(rng, 1, min(16384, _MOST_LOGITS // cols // (2 if type == "f32" else 1)))
    return {"kind": kind, "rows": rows, "cols": cols, "type": type, "masked": rng.random() < 0.4,
            "top": rng.choice((0, 1, 5, 20)) if kind == "logprob_fwd" and cols >= 32 else 0}


def _round16(n):
    return (n + 15) // 16 * 16


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rows, cols, dt = case["rows"], case["cols"], _TORCH[case["type"]]

    def normal(*shape, sigma=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(sigma).add_(mean)

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    f32, kind = torch.float32, case["kind"]
    s = {"case": case}
    if kind in ("norm_fwd", "norm_bwd", "norm_linear", "linear"):
        # features: rows of their own mean and size
        s["x"] = normal(rows, cols).mul_(normal(rows, 1).abs_().add_(0.5)).add_(normal(rows, 1, sigma=0.5)).to(dt)
    if kind in ("norm_fwd", "norm_bwd", "norm_linear"):
        s["gamma"], s["beta"] = normal(cols, sigma=0.2, mean=1.0), normal(cols, sigma=0.2)
    if kind == "norm_fwd":
        s.update(y=empty(rows, cols), mean=empty(rows, dtype=f32), rstd=empty(rows, dtype=f32))
    elif kind == "norm_bwd":
        # the statistics are what the forward pass left behind
        x = s["x"].float()
        s["mean"] = x.mean(1)
        s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + _EPS)
        s["dy"] = normal(rows, cols, sigma=0.1).to(dt)
        s.update(dx=empty(rows, cols), dgamma=empty(cols, dtype=f32), dbeta=empty(cols, dtype=f32))
    elif kind in ("linear", "norm_linear"):
        # weights were quantised when the program started: a scale for each output channel, rows padded to 16 bytes
        outs = case["outs"]
        w = normal(outs, cols, sigma=cols ** -0.5)
        s["w_scale"] = w.abs().amax(1) / 127.0
        s["w"] = torch.zeros(outs, _round16(cols), dtype=torch.int8, device="cuda")
        s["w"][:, :cols] = torch.round(w / s["w_scale"][:, None]).to(torch.int8)
        s["bias"] = normal(outs, sigma=0.1)
        s.update(q=empty(rows, _round16(cols), dtype=torch.int8), scale=empty(rows, dtype=f32), y=empty(rows, outs))
    else:
        x = normal(rows, cols, sigma=2.5)
        s["target"] = torch.randint(0, cols, (rows,), generator=g, device="cuda")
        x.scatter_add_(1, s["target"][:, None], normal(rows, 1, sigma=2.0, mean=4.0))
        if case["masked"]:
            # tokens that the grammar of the answer rules out, padding rows without a token, and one row with nothing left
            x.masked_fill_(torch.rand(rows, cols, generator=g, device="cuda") < 0.3, -_INF)
            x[rows // 2] = -_INF
            s["target"].masked_fill_(torch.rand(rows, generator=g, device="cuda") < 0.1, -1)
        s["x"] = x.to(dt)
        s["lse"], s["entropy"] = empty(rows, dtype=f32), empty(rows, dtype=f32)
        if kind == "logprob_fwd":
            s.update(logp=empty(rows, dtype=f32), top_id=empty(rows, case["top"], dtype=torch.int64), top_logp=empty(rows, case["top"], dtype=f32))
        else:
            # what the forward pass left behind, and the gradients that reach its outputs
            x = s["x"].float()
            m = x.amax(1, keepdim=True).clamp_(min=-3e38)
            e = torch.exp(x - m)
            z = e.sum(1)
            s["lse"] = m[:, 0] + torch.log(z)
            s["entropy"] = torch.where(z > 0, torch.log(z) - (e * (x - m).clamp_(min=-3e38)).sum(1) / z, 0.0)
            s["g_logp"], s["g_entropy"] = normal(rows, mean=-1.0, sigma=0.1) / rows, normal(rows, sigma=0.1) / rows
            s["dx"] = empty(rows, cols)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------


def _plain_norm(x, gamma, beta):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + _EPS)
    return (x - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def _plain_norm_bwd(s):
    x, dy = s["x"].float(), s["dy"].float()
    xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["gamma"]
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx.to(s["x"].dtype), (dy * xh).sum(0), dy.sum(0)


def _plain_linear(s, x):
    x = x.float()
    scale = (x.abs().amax(1, keepdim=True) * (1.0 / 127.0)).clamp(min=2.0 ** -126)
    q = torch.round(x * torch.reciprocal(scale))
    y = (q @ s["w"][:, : x.shape[1]].float().t()) * (scale * s["w_scale"]) + s["bias"]
    return (torch.relu(y) if s["case"]["relu"] else y).to(s["x"].dtype)


def _plain_logprob(s):
    x, target, top = s["x"].float(), s["target"], s["case"]["top"]
    m = x.amax(1, keepdim=True)
    some = m > -_INF
    e = torch.exp(x - torch.where(some, m, 0.0))
    z = e.sum(1, keepdim=True)
    lse = torch.where(some, m + torch.log(z), -_INF)
    entropy = torch.where(some, lse - torch.where(e > 0, e * x, 0.0).sum(1, keepdim=True) / z, 0.0)
    given = x.gather(1, target.clamp(min=0)[:, None])
    logp = torch.where(some, given - lse, -_INF)[:, 0]
    logp = torch.where(target < 0, 0.0, logp)
    # the likeliest tokens: by value, and by the lower index where values are equal
    bits = (x + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64) * 2 ** 32 + (2 ** 31 - torch.arange(x.shape[1], device=x.device))
    ids = 2 ** 31 - torch.topk(key, top, dim=1).values % 2 ** 32
    return logp, lse[:, 0], entropy[:, 0], ids, torch.where(some, x.gather(1, ids) - lse, -_INF)


def _plain_logprob_bwd(s):
    x, target = s["x"].float(), s["target"][:, None]
    some = (s["lse"] > -_INF)[:, None]
    lp = x - torch.where(some, s["lse"][:, None], 0.0)
    p = torch.exp(lp)
    hit = torch.arange(x.shape[1], device=x.device) == target
    g = torch.where(target >= 0, s["g_logp"][:, None], 0.0)
    dx = g * (hit.float() - p) - s["g_entropy"][:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    return torch.where(some, dx, 0.0).to(s["x"].dtype)


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "norm_fwd":
        y, mean, rstd = _plain_norm(s["x"], s["gamma"], s["beta"])
        return y.to(s["x"].dtype), mean, rstd
    if kind == "norm_bwd":
        return _plain_norm_bwd(s)
    if kind == "linear":
        return _plain_linear(s, s["x"])
    if kind == "norm_linear":
        return _plain_linear(s, _plain_norm(s["x"], s["gamma"], s["beta"])[0].to(s["x"].dtype))
    return _plain_logprob(s) if kind == "logprob_fwd" else _plain_logprob_bwd(s)


# ---- the framework's operators ---------------------------------------------------------------------------------------


def _plan(s):
    """The descriptors and the workspace that a program makes once for its sizes and keeps."""
    from paper_1611_06945_amd import binding as B

    c = s["case"]
    kind, rows, cols = c["kind"], c["rows"], c["cols"]
    dt = {"f32": B.CONV_F32, "f16": B.CONV_F16, "bf16": B.CONV_BF16}[c["type"]]
    need = 0
    if kind in ("norm_fwd", "norm_bwd"):
        s["desc"] = B.make_norm_desc(rows, cols, dt, eps=_EPS)
        need = B.layernorm_bwd_workspace_bytes(s["desc"]) if kind == "norm_bwd" else 0
    elif kind in ("linear", "norm_linear"):
        s["desc"] = B.make_int_linear_desc(rows, c["outs"], cols, dt, relu=c["relu"])
        s["in_desc"] = B.make_quant_desc(rows, cols, dt) if kind == "linear" else B.make_norm_desc(rows, cols, dt, eps=_EPS, ldy=_round16(cols))
        need = B.int_linear_workspace_bytes(s["desc"])
    else:
        s["desc"] = B.make_logprob_desc(rows, cols, dt, top=c["top"])
        need = B.logprob_workspace_bytes(s["desc"]) if kind == "logprob_fwd" else 0
    s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    s["B"] = B


def _own(s):
    if "B" not in s:
        _plan(s)
    B, kind, ws = s["B"], s["case"]["kind"], s["ws"]
    if kind == "norm_fwd":
        B.layernorm_fwd(s["desc"], s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"])
        return s["y"], s["mean"], s["rstd"]
    if kind == "norm_bwd":
        B.layernorm_bwd(s["desc"], s["x"], s["dy"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], ws, ws.numel())
        return s["dx"], s["dgamma"], s["dbeta"]
    if kind in ("linear", "norm_linear"):
        if kind == "linear":
            B.quantize_rows(s["in_desc"], s["x"], s["q"], s["scale"])
        else:
            B.layernorm_quant_fwd(s["in_desc"], s["x"], s["gamma"], s["beta"], s["q"], s["scale"])
        B.int_linear_fwd(s["desc"], s["q"], s["scale"], s["w"], s["w_scale"], s["bias"], s["y"], ws, ws.numel())
        return s["y"]
    if kind == "logprob_fwd":
        B.logprob_fwd(s["desc"], s["x"], s["target"], s["logp"], s["lse"], s["entropy"], s["top_id"], s["top_logp"], ws, ws.numel())
        return s["logp"], s["lse"], s["entropy"], s["top_id"], s["top_logp"]
    B.logprob_bwd(s["desc"], s["x"], s["target"], s["lse"], s["entropy"], s["g_logp"], s["g_entropy"], s["dx"])
    return s["dx"]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    t, d, es = case["rows"], case["cols"], _BYTES[case["type"]]
    kind = case["kind"]
    if kind == "norm_fwd":
        return {"bytes": 2 * t * d * es + 8 * d + 8 * t, "flops": 8 * t * d}
    if kind == "norm_bwd":
        return {"bytes": 3 * t * d * es + 12 * d + 8 * t, "flops": 14 * t * d}
    if kind in ("linear", "norm_linear"):
        n = case["outs"]
        return {"bytes": t * d * es + n * d + 8 * n + t * n * es + (8 * d if kind == "norm_linear" else 0), "flops": 2 * t * d * n}
    if kind == "logprob_fwd":
        return {"bytes": t * d * es + t * (8 + 12 + 12 * case["top"]), "flops": 6 * t * d}
    return {"bytes": 2 * t * d * es + t * 24, "flops": 8 * t * d}


# ---- from the definitions, in 64 bits --------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    kind, d = case["kind"], case["cols"]
    x = s["x"].double()
    if kind in ("norm_fwd", "norm_linear"):
        mean = x.sum(1) / d
        var = ((x - mean[:, None]) ** 2).sum(1) / d
        rstd = 1.0 / torch.sqrt(var + _EPS)
        y = s["gamma"].double() * ((x - mean[:, None]) * rstd[:, None]) + s["beta"].double()
        if kind == "norm_fwd":
            return y, mean, rstd
        x = y
    if kind in ("linear", "norm_linear"):
        # the codes are part of the operator's definition: whole multiples of a 127th of the row's largest value
        step = x.abs().max(1).values / 127.0
        codes = torch.round(x / step[:, None])
        w = s["w"][:, :d].double() * s["w_scale"].double()[:, None]
        y = torch.matmul(codes * step[:, None], w.t().contiguous()) + s["bias"].double()
        return torch.clamp(y, min=0.0) if case["relu"] else y
    if kind == "norm_bwd":
        # through the centred and scaled rows: dx = rstd (g - the parts of g along 1 and along xh)
        xh = (x - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
        dy = s["dy"].double()
        g = dy * s["gamma"].double()
        along_one, along_xh = g.sum(1) / d, (g * xh).sum(1) / d
        dx = (g - along_one[:, None] - along_xh[:, None] * xh) * s["rstd"].double()[:, None]
        return dx, (dy * xh).sum(0), dy.sum(0)
    if kind == "logprob_fwd":
        lse = torch.logsumexp(x, 1)
        empty = lse == -_INF
        p = torch.exp(x - lse[:, None]).masked_fill_(empty[:, None], 0.0)
        info = (lse[:, None] - x).masked_fill_(p == 0, 0.0)
        entropy = (p * info).sum(1)
        logp = torch.take_along_dim(x, s["target"].clamp(min=0)[:, None], 1)[:, 0] - lse
        logp = logp.masked_fill(empty, -_INF).masked_fill(s["target"] < 0, 0.0)
        top = torch.sort(x, dim=1, descending=True).values[:, : case["top"]] - lse[:, None]
        return logp, lse, entropy, None, top.masked_fill(empty[:, None], -_INF)
    lse, h = s["lse"].double()[:, None], s["entropy"].double()[:, None]
    empty = lse == -_INF
    p = torch.exp(x - lse.masked_fill(empty, 0.0)).masked_fill_(empty, 0.0)
    glp = s["g_logp"].double().masked_fill(s["target"] < 0, 0.0)[:, None]
    info = (lse - x).masked_fill_(p == 0, 0.0)
    dx = p * (s["g_entropy"].double()[:, None] * (info - h) - glp)
    at = s["target"].clamp(min=0)[:, None]
    return dx.scatter_add_(1, at, glp.masked_fill(empty, 0.0))
