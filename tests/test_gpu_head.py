"""The operators on rows run together: the scoring head in 8 bits and the training head against the same layers in 64 bits, on
streams, from threads, and from a recorded graph."""
import threading

import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl
from paper_1611_06945_amd.head import ScoringHead, TrainingHead, demo

from gpu_util import torch_mod
from rows_util import ROUND, stored, torch_type

pytestmark = pytest.mark.gpu


def case(T, D, V, dtype, seed):
    torch = torch_mod()
    rng = np.random.default_rng(seed)
    c = {"x": stored(rng.normal(size=(T, D)) * 2 + 0.5, dtype), "w": stored(rng.normal(size=(V, D)) * 2 * D ** -0.5, dtype),
         "gamma": rng.normal(1, 0.2, D).astype(np.float32).astype(np.float64), "beta": rng.normal(0, 0.2, D).astype(np.float32).astype(np.float64),
         "bias": rng.normal(0, 0.2, V).astype(np.float32).astype(np.float64), "target": rng.integers(0, V, T)}
    d = {k: torch.from_numpy(c[k]).cuda().to(torch_type(dtype)) for k in ("x", "w")}
    d.update({k: torch.from_numpy(c[k].astype(np.float32)).cuda() for k in ("gamma", "beta", "bias")})
    d["target"] = torch.from_numpy(c["target"]).cuda()
    return c, d


@pytest.mark.parametrize("dtype", [wl.F32, wl.F16, wl.BF16])
@pytest.mark.parametrize("T,D,V", [(1, 64, 1000), (20, 384, 1000), (3, 100, 9001), (130, 256, 333)])
def test_scoring_head(T, D, V, dtype):
    """The 8-bit layers' logits as stored, then the exact operators: the head's answers are those of its own logits; the logits
    are those of the unquantised layers within the error of the 8-bit codes."""
    c, d = case(T, D, V, dtype, T)
    head = ScoringHead(d["gamma"], d["beta"], d["w"], d["bias"], max_rows=T + 3, top=5)
    r = head.score(d["x"], d["target"])
    logits = head.logits[:T].double().cpu().numpy()
    want = ro.logprob(logits, c["target"], 5)
    for k in ("logp", "lse", "entropy", "top_logp"):
        assert np.allclose(r[k].cpu().numpy(), want[k], atol=2e-5, rtol=2e-5), k
    assert np.array_equal(r["top_id"].cpu().numpy(), want["top_id"])
    y = ro.layernorm(c["x"], c["gamma"], c["beta"], 1e-5)[0]
    exact = y @ c["w"].T + c["bias"]
    # a code is off by half a step of amax / 127 at most on either side; the roundings of a row's products are independent, of
    # random sign: six standard deviations of sum(dy w + y dw) over D, and the storage type's roundings of y and of the logits
    step_y, step_w = np.abs(y).max(1) / 127, np.abs(c["w"]).max(1) / 127
    sd = np.sqrt((step_y ** 2 / 12)[:, None] * (c["w"] ** 2).sum(1)[None] + (step_w ** 2 / 12)[None] * (y ** 2).sum(1)[:, None]
                 + ROUND[dtype] ** 2 * (y ** 2) @ (c["w"] ** 2).T)
    off = np.abs(logits - exact)
    assert (off > 6 * sd + ROUND[dtype] * np.abs(exact) + 1e-5).sum() <= 1e-6 * off.size
    assert head.score(d["x"])["logp"] is None


@pytest.mark.parametrize("dtype", [wl.F32, wl.F16])
@pytest.mark.parametrize("T,D,V", [(1, 32, 10), (48, 96, 1000), (33, 100, 130)])
def test_training_head(T, D, V, dtype):
    c, d = case(T, D, V, dtype, T + D)
    torch = torch_mod()
    head = TrainingHead(T, D, V, torch_type(dtype))
    logp, entropy = head.forward(d["x"], d["gamma"], d["beta"], d["w"], d["target"])
    rng = np.random.default_rng(5)
    gl, gh = rng.normal(size=T).astype(np.float32), rng.normal(size=T).astype(np.float32)
    y, mean, rstd = ro.layernorm(c["x"], c["gamma"], c["beta"], 1e-5)
    logits = y @ c["w"].T
    r = ro.logprob(logits, c["target"], 0)
    # activations and logits are stored in 8 or 11 or 24 bits: errors relative to each tensor's size, a few roundings deep
    u = 8 * ROUND[dtype] + 2e-5

    def near(got, want, what):
        got = got.double().cpu().numpy()
        assert np.linalg.norm(got - want) <= u * np.linalg.norm(want) + u * 1e-3, what

    near(logp, r["logp"], "logp")
    near(entropy, r["entropy"], "entropy")
    dx, dgamma, dbeta, dw = head.backward(torch.from_numpy(gl).cuda(), torch.from_numpy(gh).cuda())
    dl = ro.logprob_bwd(logits, c["target"], r["lse"], r["entropy"], gl.astype(np.float64), gh.astype(np.float64))
    want_dx, want_dg, want_db = ro.layernorm_bwd(c["x"], dl @ c["w"], c["gamma"], mean, rstd)
    near(dw, dl.T @ y, "dweight")
    near(dx, want_dx, "dfeatures")
    near(dgamma, want_dg, "dgamma")
    near(dbeta, want_db, "dbeta")


def test_demo_learns_and_the_8_bit_head_agrees():
    first, last, hit = demo(rows=256, D=128, V=200, steps=30, log=lambda *_: None)
    assert last > first + 2.0 and hit > 0.95


def test_scoring_on_streams_from_threads_equals_the_serial_calls():
    torch = torch_mod()
    shapes = [(1, 512, 20000), (20, 384, 1000), (64, 100, 3001), (300, 256, 700)]
    jobs = [(ScoringHead(d["gamma"], d["beta"], d["w"], d["bias"], max_rows=s[0], top=5), d) for s, (_, d) in ((s, case(*s, wl.F16, 40 + i)) for i, s in enumerate(shapes))]
    serial = [{k: v.clone() for k, v in h.score(d["x"], d["target"]).items()} for h, d in jobs]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        h, d = jobs[i]
        stream = torch.cuda.Stream()
        for _ in range(20):
            r = h.score(d["x"], d["target"], stream)
            stream.synchronize()
            if not all(torch.equal(r[k], serial[i][k]) for k in serial[i]):
                bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


@pytest.mark.parametrize("T,D,V", [(1, 256, 40000), (20, 384, 1000)])
def test_scoring_head_in_a_graph(T, D, V):
    torch = torch_mod()
    _, d = case(T, D, V, wl.BF16, 9)
    head = ScoringHead(d["gamma"], d["beta"], d["w"], max_rows=T, top=5)
    x, target = d["x"].clone(), d["target"].clone()
    head.plan(T, D)
    head.score(x, target)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = head.score(x, target)
    for seed in range(5):
        c2, d2 = case(T, D, V, wl.BF16, 90 + seed)
        x.copy_(d2["x"]), target.copy_(d2["target"])
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        eager = head.score(x, target)
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], eager[k]) for k in got), seed


def test_refusals_of_the_heads_own():
    _, d = case(4, 64, 100, wl.F16, 1)
    head = ScoringHead(d["gamma"], d["beta"], d["w"], max_rows=4, top=3)
    for x in (d["x"].float(), d["x"][:, :32], torch_mod().cat([d["x"], d["x"]])):
        with pytest.raises(ValueError):
            head.score(x)
    with pytest.raises(B.ConvError):
        ScoringHead(d["gamma"], d["beta"], d["w"], max_rows=4, top=101).score(d["x"])


def test_a_recorded_graph_outlives_scores_of_other_sizes():
    """One row is recorded; batches of sizes that need more workspace are scored and memory is taken in between; the graph still
    writes only to the head's own buffers."""
    torch = torch_mod()
    D, V = 256, 50257
    _, d = case(20, D, V, wl.BF16, 31)
    head = ScoringHead(d["gamma"], d["beta"], d["w"], max_rows=20, top=5)
    x, target = d["x"][:1].clone(), d["target"][:1].clone()
    head.score(x, target)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = head.score(x, target)
    want = []
    for i in range(20):
        want.append({k: v.clone() for k, v in head.score(d["x"][i:i + 1], d["target"][i:i + 1]).items()})
    held = []
    for i, rows in enumerate((2, 4, 8, 20, 3, 1)):
        head.score(d["x"][:rows], d["target"][:rows])
        held += [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for n in (256, 768, 1536, 6144, 12288)]
        x.copy_(d["x"][i:i + 1]), target.copy_(d["target"][i:i + 1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[i][k]) for k in out), i
        assert all(bool((h == 77).all()) for h in held), i


def test_one_row_out_of_a_channel_plane():
    """The features of one image as a slice of its channel planes are refused, as those of two are; made dense they are scored."""
    torch = torch_mod()
    _, d = case(1, 64, 100, wl.F16, 3)
    head = ScoringHead(d["gamma"], d["beta"], d["w"], max_rows=4, top=3)
    planes = torch.zeros(1, 64, 2, 2, dtype=torch.float16, device="cuda")
    planes[:, :, 0, 0] = d["x"]
    with pytest.raises(ValueError):
        head.score(planes[:, :, 0, 0])
    got = {k: v.clone() for k, v in head.score(planes[:, :, 0, 0].contiguous(), d["target"]).items()}
    want = head.score(d["x"], d["target"])
    assert all(torch.equal(got[k], want[k]) for k in got)


@pytest.mark.parametrize("T,D,V", [(1, 32, 10), (48, 96, 1000), (33, 100, 130), (300, 384, 1000)])
def test_training_head_in_bf16(T, D, V):
    """Tensors on the way (the normalised rows y, the logits z, their gradient dz, the product dy = dz w) are stored in bf16, so each
    carries an error of 2^-8 of an element; what follows is linear in them but for the softmax.  Bounds in the 2-norm: u = 2^-8,
    du(t) the norm of t's stored error."""
    c, d = case(T, D, V, wl.BF16, 3 * T + D)
    torch = torch_mod()
    head = TrainingHead(T, D, V, torch.bfloat16)
    rng = np.random.default_rng(6)
    gl, gh = rng.normal(size=T).astype(np.float32), rng.normal(size=T).astype(np.float32)
    head.forward(d["x"], d["gamma"], d["beta"], d["w"], d["target"])
    # what the head stored, taken as the exact inputs of the next step: each step is held to its own roundings
    y = head.y.double().cpu().numpy()
    z = head.logits.double().cpu().numpy()
    u, n, f32 = 2.0 ** -8, np.linalg.norm, 2.0 ** -24
    want_y, mean, rstd = ro.layernorm(c["x"], c["gamma"], c["beta"], 1e-5)
    assert (np.abs(y - want_y) <= u * np.abs(want_y) + 1e-4).all()
    want_z = y @ c["w"].T
    assert (np.abs(z - want_z) <= 1.01 * u * np.abs(want_z) + (D + 8) * f32 * (np.abs(y) @ np.abs(c["w"]).T) + 1e-6).all()
    r = ro.logprob(z, c["target"], 0)
    assert np.allclose(head.logp.cpu().numpy(), r["logp"], atol=2e-5, rtol=2e-5) and np.allclose(head.entropy.cpu().numpy(), r["entropy"], atol=5e-5, rtol=5e-5)
    dx, dgamma, dbeta, dw = head.backward(torch.from_numpy(gl).cuda(), torch.from_numpy(gh).cuda())
    dz = head.logits.double().cpu().numpy()
    want_dz = ro.logprob_bwd(z, c["target"], r["lse"], r["entropy"], gl.astype(np.float64), gh.astype(np.float64))
    p = np.exp(z - r["lse"][:, None])
    size = p * (np.abs(gl)[:, None] + np.abs(gh)[:, None] * (np.abs(z - r["lse"][:, None]) + r["entropy"][:, None] + 1))
    assert (np.abs(dz - want_dz) <= 1.01 * u * np.abs(want_dz) + 1e-4 * size + 1e-30).all()
    dy = head.dy.double().cpu().numpy()
    near = lambda got, a, b, k: (np.abs(got - a @ b) <= 1.01 * u * np.abs(a @ b) + (k + 8) * f32 * (np.abs(a) @ np.abs(b)) + 1e-30).all()  # noqa: E731
    assert near(dy, dz, c["w"], V)
    assert near(dw.double().cpu().numpy(), dz.T, y, T)
    want_dx, want_dg, want_db = ro.layernorm_bwd(c["x"], dy, c["gamma"], mean, rstd)
    # (statistics of 32 bits: a part in 10^5 of the sizes that enter, as in the layers' own tests)
    xh = np.abs((c["x"] - mean[:, None]) * rstd[:, None])
    g = np.abs(dy * c["gamma"])
    sizes = rstd[:, None] * (g + g.mean(1)[:, None] + xh * (g * xh).mean(1)[:, None])
    assert (np.abs(dx.double().cpu().numpy() - want_dx) <= 1.01 * u * np.abs(want_dx) + 1e-5 * sizes).all()
    assert (np.abs(dgamma.double().cpu().numpy() - want_dg) <= 1e-5 * (np.abs(dy) * (xh + 1)).sum(0) + 1e-30).all()
    assert (np.abs(dbeta.double().cpu().numpy() - want_db) <= 1e-5 * np.abs(dy).sum(0) + 1e-30).all()
    # and the whole of it near the gradients without any rounding: a few roundings deep
    full = ro.logprob_bwd(want_y @ c["w"].T, c["target"], *(ro.logprob(want_y @ c["w"].T, c["target"], 0)[k] for k in ("lse", "entropy")), gl.astype(np.float64), gh.astype(np.float64))
    want = full.T @ want_y
    assert n(dw.double().cpu().numpy() - want) <= 0.1 * n(want)


def test_a_new_head_scores_on_any_stream():
    """The weights are quantised when the head is made; a first score on another stream finds them done."""
    torch = torch_mod()
    _, d = case(8, 512, 30000, wl.F16, 77)
    want = {k: v.clone() for k, v in ScoringHead(d["gamma"], d["beta"], d["w"], max_rows=8, top=5).score(d["x"], d["target"]).items()}
    busy = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        for _ in range(20):
            busy = torch.tanh(busy @ busy)  # the current stream is behind
        head = ScoringHead(d["gamma"], d["beta"], d["w"], max_rows=8, top=5)
        got = head.score(d["x"], d["target"], side)
        side.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)
