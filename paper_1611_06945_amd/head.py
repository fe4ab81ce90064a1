"""The end of a classifier or of a network that answers with tokens, on the operators on rows of the C ABI.

    features [T][D] -> layer norm -> product with a weight [V][D] -> log probabilities

`ScoringHead` is the serving form: the layer norm writes 8-bit rows, the product multiplies them with weights that were
quantised when the head was made, and the answers are log probabilities of given tokens, entropies and the likeliest
alternatives.  It allocates everything up front, for any number of rows up to its own, so a call is three launches (four or five
for few rows of a long vocabulary) and can be recorded into a HIP graph.

`TrainingHead` is the training form of the same layers in their storage type: log probabilities and entropies of a batch, and
the gradients of  sum_t g_logp[t] logp[t] + g_entropy[t] entropy[t]  in the features, gamma, beta and the weight (there is no bias).  Its dense products
are the library's 1x1 convolutions: T rows are T images of one pixel, and the two products of the backward pass are convolutions of
transposed tensors.

    python -m paper_1611_06945_amd.head            # trains a small head on synthetic features, then scores in 8 bits
"""
from __future__ import annotations

from . import binding as B

GPU = "cuda"  # where every tensor here lives


def _code(torch, dtype):
    return {torch.float32: B.CONV_F32, torch.float16: B.CONV_F16, torch.bfloat16: B.CONV_BF16}[dtype]


def _check(name, t, dtype, shape, device):
    """The kernels are handed addresses: a tensor of another type, size, layout or place would be read as what it is not."""
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError("%s must be %s %s, dense, on %s; it is %s %s with strides %s on %s" % (
            name, dtype, list(shape), device, t.dtype, list(t.shape), list(t.stride()), t.device))


class ScoringHead:
    def __init__(self, gamma, beta, weight, bias=None, max_rows: int = 64, top: int = 5, eps: float = 1e-5, logits_dtype=None):
        """gamma, beta: fp32 [D] or None; weight: [V][D] in fp32, fp16 or bf16 on the GPU, which is also the type of the
        features; bias: fp32 [V] or None.  `logits_dtype`: storage type of the logits (default: the weight's)."""
        import torch

        self.torch, self.gamma, self.beta, self.bias, self.eps = torch, gamma, beta, bias, eps
        self.V, self.D = weight.shape
        if self.D > 1 and weight.stride(1) != 1:
            raise ValueError("the columns of a weight's row have to be next to each other")
        if weight.device.type != GPU:
            raise ValueError("the weight is on %s, not on the GPU" % weight.device)
        for name, t, n in (("gamma", gamma, self.D), ("beta", beta, self.D), ("bias", bias, self.V)):
            if t is not None:
                _check(name, t, torch.float32, (n,), weight.device)
        self.max_rows, self.top = int(max_rows), int(top)
        self.code, self.logits_dtype = _code(torch, weight.dtype), logits_dtype or weight.dtype
        self.dtype = weight.dtype
        dev, ld = weight.device, B.row_stride(self.D)
        self.w = torch.empty(self.V, ld, dtype=torch.int8, device=dev)
        self.w_scale = torch.empty(self.V, dtype=torch.float32, device=dev)
        B.quantize_rows(B.make_quant_desc(self.V, self.D, self.code, weight.stride(0) if self.V > 1 else self.D), weight, self.w, self.w_scale)
        f32 = dict(dtype=torch.float32, device=dev)
        self.q, self.q_scale = torch.empty(self.max_rows, ld, dtype=torch.int8, device=dev), torch.empty(self.max_rows, **f32)
        self.logits = torch.empty(self.max_rows, self.V, dtype=self.logits_dtype, device=dev)
        self.logp, self.lse, self.entropy = (torch.empty(self.max_rows, **f32) for _ in range(3))
        self.top_id = torch.empty(self.max_rows, self.top, dtype=torch.int64, device=dev)
        self.top_logp = torch.empty(self.max_rows, self.top, **f32)
        # One workspace for the head's whole life: recorded graphs and calls on other streams hold its address.  What is needed goes up
        # and down with the rows (workgroups that share a row or a reduction become fewer), so every number of them is asked.
        need = 256
        for rows in range(1, self.max_rows + 1):
            linear, logprob = self._products(rows)
            need = max(need, B.int_linear_workspace_bytes(linear), B.logprob_workspace_bytes(logprob))
        self._plans, self._ws = {}, torch.empty(need, dtype=torch.uint8, device=dev)
        if GPU == "cuda" and not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(dev).synchronize()  # the 8-bit weights are there for whatever stream scores first

    def _products(self, rows: int):
        code = _code(self.torch, self.logits_dtype)
        return (B.make_int_linear_desc(rows, self.V, self.D, code, lda=self.q.stride(0), ldw=self.w.stride(0)),
                B.make_logprob_desc(rows, self.V, code, self.top))

    def plan(self, rows: int, ldx: int):
        """The three descriptors for a number of rows and a row stride of the features, and the answers' places, made once."""
        if not 0 <= rows <= self.max_rows:
            raise ValueError("a head of %d rows cannot score %d" % (self.max_rows, rows))
        key = (rows, ldx)
        if key not in self._plans:
            answers = {k: getattr(self, k)[:rows] for k in ("logp", "lse", "entropy", "top_id", "top_logp")}
            self._plans[key] = (B.make_norm_desc(rows, self.D, self.code, self.eps, ldx, self.q.stride(0)), *self._products(rows), answers)
        return self._plans[key]

    def score(self, features, target=None, stream=None):
        """features [T][D] (rows may be strided), target int64 [T] or None (negative: no token).  Returns views of the head's own
        buffers, valid until the next call: logp (None without target), lse, entropy, top_id, top_logp.  Calls of one head share
        its buffers, so on several streams they have to be put in order."""
        rows = features.shape[0]
        if features.device != self.w.device:
            raise ValueError("the features are on %s, the head on %s" % (features.device, self.w.device))
        if features.shape[1] != self.D or features.dtype != self.dtype or (rows and self.D > 1 and features.stride(1) != 1) or rows > self.max_rows:
            raise ValueError("features must be [T <= %d][%d] of %s, the columns of a row next to each other" % (self.max_rows, self.D, self.dtype))
        if target is not None:
            _check("target", target, self.torch.int64, (rows,), self.w.device)
        norm, linear, logprob, answers = self.plan(rows, features.stride(0) if rows > 1 else self.D)
        ws, n = self._ws, self._ws.numel()
        B.layernorm_quant_fwd(norm, features, self.gamma, self.beta, self.q, self.q_scale, stream)
        B.int_linear_fwd(linear, self.q, self.q_scale, self.w, self.w_scale, self.bias, self.logits, ws, n, stream)
        logp = None if target is None else self.logp
        tops = (self.top_id, self.top_logp) if self.top else (None, None)
        B.logprob_fwd(logprob, self.logits, target, logp, self.lse, self.entropy, *tops, ws, n, stream)
        return dict(answers) if logp is not None else {**answers, "logp": None}


class TrainingHead:
    def __init__(self, rows: int, D: int, V: int, dtype, eps: float = 1e-5, device="cuda"):
        """Buffers and descriptors for batches of `rows` features [rows][D] over V tokens, in `dtype`."""
        import torch

        if torch.device(device).type != GPU:
            raise ValueError("a head on %s: its kernels run on the GPU" % device)
        self.torch, self.rows, self.D, self.V, self.dtype = torch, rows, D, V, dtype
        self.code = _code(torch, dtype)
        new = lambda *shape: torch.empty(*shape, dtype=dtype, device=device)  # noqa: E731
        vec = lambda n: torch.empty(n, dtype=torch.float32, device=device)  # noqa: E731
        self.y, self.dy, self.y_t = new(rows, D), new(rows, D), new(D, rows)
        self.logits, self.dlogits_t, self.w_t = new(rows, V), new(V, rows), new(D, V)
        self.dx, self.dw = new(rows, D), new(V, D)
        self.mean, self.rstd, self.logp, self.lse, self.entropy = (vec(rows) for _ in range(5))
        self.dgamma, self.dbeta = vec(D), vec(D)
        self.norm = B.make_norm_desc(rows, D, self.code, eps)
        self.logprob = B.make_logprob_desc(rows, V, self.code)
        product = lambda n, c, k: B.make_desc(n, c, 1, 1, k, 1, 1, dtype=self.code)  # noqa: E731
        self.to_logits, self.to_dy, self.to_dw = product(rows, D, V), product(rows, V, D), product(V, rows, D)
        need = max([B.layernorm_bwd_workspace_bytes(self.norm), B.logprob_workspace_bytes(self.logprob)] +
                   [B.conv_workspace_bytes(d) for d in (self.to_logits, self.to_dy, self.to_dw)])
        self.ws = torch.empty(max(256, need), dtype=torch.uint8, device=device)
        self.saved = None

    def forward(self, features, gamma, beta, weight, target, stream=None):
        """features [rows][D] and weight [V][D] of the head's type, gamma and beta fp32 [D] or None, target int64 [rows], all dense
        -> (logp, entropy) of the batch, fp32 [rows]; keeps what backward() needs.  There is no bias."""
        f32, dev = self.torch.float32, self.logits.device
        for name, t, dtype, shape in (("features", features, self.dtype, (self.rows, self.D)), ("gamma", gamma, f32, (self.D,)), ("beta", beta, f32, (self.D,)),
                                      ("weight", weight, self.dtype, (self.V, self.D)), ("target", target, self.torch.int64, (self.rows,))):
            if t is not None:
                _check(name, t, dtype, shape, dev)
        ws, n = self.ws, self.ws.numel()
        self.saved = None
        B.layernorm_fwd(self.norm, features, gamma, beta, self.y, self.mean, self.rstd, stream)
        B.conv_fwd_ws(self.to_logits, self.y, weight, None, self.logits, ws, n, stream)
        B.logprob_fwd(self.logprob, self.logits, target, self.logp, self.lse, self.entropy, None, None, ws, n, stream)
        self.saved = (features, gamma, weight, target)
        return self.logp, self.entropy

    def backward(self, g_logp, g_entropy=None, stream=None):
        """g_logp, g_entropy: fp32 [rows], one may be None -> (dfeatures, dgamma, dbeta, dweight).  Once for each forward(), since the
        logits' gradient takes the logits' place: give both gradients to one call.  Features, gamma and weight have to be those of
        forward() still."""
        if self.saved is None:
            raise RuntimeError("backward() needs a forward() of its own: the logits are no longer there")
        for name, t in (("g_logp", g_logp), ("g_entropy", g_entropy)):
            if t is not None:
                _check(name, t, self.torch.float32, (self.rows,), self.logits.device)
        features, gamma, weight, target = self.saved
        ws, n = self.ws, self.ws.numel()
        B.logprob_bwd(self.logprob, self.logits, target, self.lse, self.entropy, g_logp, g_entropy, self.logits, stream)
        self.saved = None
        B.conv_convert_layout(1, self.V, self.D, self.code, weight, self.w_t, stream)
        B.conv_fwd_ws(self.to_dy, self.logits, self.w_t, None, self.dy, ws, n, stream)
        B.conv_convert_layout(1, self.rows, self.V, self.code, self.logits, self.dlogits_t, stream)
        B.conv_convert_layout(1, self.rows, self.D, self.code, self.y, self.y_t, stream)
        B.conv_fwd_ws(self.to_dw, self.dlogits_t, self.y_t, None, self.dw, ws, n, stream)
        B.layernorm_bwd(self.norm, features, self.dy, gamma, self.mean, self.rstd, self.dx, self.dgamma, self.dbeta, ws, n, stream)
        return self.dx, self.dgamma, self.dbeta, self.dw


def demo(rows: int = 512, D: int = 384, V: int = 1000, steps: int = 40, rate: float = 4.0, log=print):
    """Trains the head on features around one random centre a class, then scores the same features in 8 bits; returns the mean
    log probabilities before and after, and how often the 8-bit head's first alternative is the class."""
    import torch

    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    centres = torch.randn(V, D, generator=g, device="cuda")
    target = torch.randint(0, V, (rows,), generator=g, device="cuda")
    x = (centres[target] + 0.3 * torch.randn(rows, D, generator=g, device="cuda")).half()
    w = (torch.randn(V, D, generator=g, device="cuda") * D ** -0.5)
    gamma, beta = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    head = TrainingHead(rows, D, V, torch.float16)
    # loss = -mean logp; its gradient is scaled by 256 for fp16 and scaled back where the weights are moved
    g_logp = torch.full((rows,), -256.0 / rows, device="cuda")
    seen = []
    for step in range(steps):
        logp, entropy = head.forward(x, gamma, beta, w.half(), target)
        seen.append(float(logp.mean()))
        _, dgamma, dbeta, dw = head.backward(g_logp)
        for p, d in ((w, dw), (gamma, dgamma), (beta, dbeta)):
            p.sub_(d.float() * (rate / 256))
        if step % 10 == 0 or step == steps - 1:
            log("step %3d: mean log probability %8.4f, mean entropy %.4f" % (step, seen[-1], float(entropy.mean())))
    scores = ScoringHead(gamma, beta, w.half(), max_rows=rows, top=5).score(x, target)
    hit = float((scores["top_id"][:, 0] == target).float().mean())
    log("8-bit head: mean log probability %.4f, first alternative is the class %.1f %%, among the five %.1f %%" % (
        float(scores["logp"].mean()), 100 * hit, 100 * float((scores["top_id"] == target[:, None]).any(1).float().mean())))
    return seen[0], seen[-1], hit


if __name__ == "__main__":
    demo()
