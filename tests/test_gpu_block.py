"""Blocks of rows, a head behind them and the update of their weights, together on the GPU: against 64 bits through autograd, in graphs and on streams.

Bounds on the norm of a gradient: every operator on the way adds up at most D + hidden + rows terms in fp32, and the sums of its terms' magnitudes are
at most 8 times its result here (random signs: the root of the number of terms, 12 at most, times 0.6); 16 operators lie on the longest way, errors at random signs: a quarter.  16-bit types: each stored tensor and each
result is rounded once on top, 24 of them on the way, at random signs taken for their worst half.  ReLU's slope jumps: where a sum, off by t of its size, changes its sign (a share 2 phi(0) t = 0.8 t of
normal values, phi their density) its slope is wrong by one, where half of all slopes are one: sqrt(0.8 t / 0.5) of the gradient's norm more in 16-bit types (in fp32 a handful of sums)."""
import numpy as np
import pytest

from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import block as blk
from paper_1611_06945_amd import workloads as wl
from paper_1611_06945_amd.head import TrainingHead

from gpu_util import torch_mod
from rows_util import EPS32, ROUND, torch_type

pytestmark = pytest.mark.gpu

ROWS, D, HIDDEN, V = 33, 48, 80, 20


def bound(dtype, act="gelu"):
    t = 16 * 8 * (D + HIDDEN + ROWS) * EPS32 / 4 + (12 * ROUND[dtype] if dtype != wl.F32 else 0.0)
    return t + (np.sqrt(1.6 * t) if act == "relu" and dtype != wl.F32 else 0.0)


def trunk(dtype, depth, gate_rows=0, sigmoid=False, act="gelu", rms=False, post=True, seed=0, rows=ROWS, d=D, hidden=HIDDEN):
    torch = torch_mod()
    tt = torch_type(dtype)
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks = [blk.TrainingBlock(rows, d, hidden, tt, act, rms, post, gate_rows, sigmoid, last=i == depth - 1) for i in range(depth)]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    weights = []
    for b in blocks:
        p = blk.start_weights(b, g)
        weights.append({k: v.to(tt) if k in blk.WEIGHTS else (v + 0.2 * rnd(*v.shape)) for k, v in p.items()})
    gates = [rnd(-(-rows // gate_rows), d).to(tt) if gate_rows else None for _ in blocks]
    return blocks, weights, gates, rnd(rows, d).to(tt), rnd(rows, d).to(tt)


def run(blocks, weights, gates, r, y, dr):
    for b, p, gt in zip(blocks, weights, gates):
        r, y = b.forward(r, y, p, gt)
    dy = None
    for b in reversed(blocks):
        dr, dy = b.backward(dr, dy)
    return r, dr, dy


def in_64(blocks, weights, gates, r, y, dr, act, rms, post, gate_rows, sigmoid):
    """The same through float64 autograd on the CPU: (r_out, leaves by name)."""
    torch = torch_mod()
    up = lambda t: None if t is None else t.detach().double().cpu().requires_grad_()  # noqa: E731
    leaves = {"r": up(r), "y": up(y)}
    acts = {"none": lambda z: z, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}

    def norm(x):
        x = x if rms else x - x.mean(1, keepdim=True)
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5)

    a, b = leaves["r"], leaves["y"]
    for i, (p, gt) in enumerate(zip(weights, gates)):
        q = {k: up(v) for k, v in p.items()}
        leaves.update({"%d.%s" % (i, k): v for k, v in q.items()})
        h = acts[act](b @ q["w1"].T + q["b1"]) @ q["w2"].T + q["b2"]
        u = norm(h) * q["gamma_h"] + q["beta_h"] if post else h
        if gt is not None:
            leaves["%d.gate" % i] = e = up(gt)
            e = e.repeat_interleave(gate_rows, 0)[: len(a)]
            u = u * (torch.sigmoid(e) if sigmoid else e)
        a = a + q["scale"] * u
        b = norm(a) * q["gamma"] + q["beta"] if "gamma" in q else None
    names = list(leaves)
    got = torch.autograd.grad(a, [leaves[n] for n in names], dr.double().cpu())
    return a.detach(), dict(zip(names, got))


def near(got, want, tol, what):
    got, want = got.double().cpu().numpy(), want.numpy()
    off, size = np.linalg.norm(got - want), np.linalg.norm(want)
    assert off <= tol * size, "%s: %.3g of its norm off where %.3g is allowed" % (what, off / size, tol)


@pytest.mark.parametrize("dtype", [wl.F32, wl.F16, wl.BF16])
@pytest.mark.parametrize("kind", [dict(), dict(gate_rows=7, sigmoid=True, act="silu"), dict(post=False, rms=True, act="relu", gate_rows=1), dict(rms=True)])
def test_gradients_of_a_chain(kind, dtype):
    kind = dict(dict(act="gelu", rms=False, post=True, gate_rows=0, sigmoid=False), **kind)
    blocks, weights, gates, r, y = trunk(dtype, 2, seed=3, **kind)
    dr = torch_mod().randn(ROWS, D, generator=torch_mod().Generator(device="cuda").manual_seed(9), device="cuda").to(r.dtype)
    r_out, d_r, d_y = run(blocks, weights, gates, r, y, dr)
    want_r, want = in_64(blocks, weights, gates, r, y, dr, **kind)
    near(r_out, want_r, bound(dtype), "r_out")
    tol = bound(dtype, kind["act"])
    near(d_r, want["r"], tol, "dr")
    near(d_y, want["y"], tol, "dy")
    for i, b in enumerate(blocks):
        for k in b.shapes:
            near(b.grads[k], want["%d.%s" % (i, k)], tol, "%d.%s" % (i, k))
        if b.dgate is not None:
            near(b.dgate, want["%d.gate" % i], tol, "%d.gate" % i)


def test_a_chain_with_a_head_in_a_graph():
    """Forward, backward and update recorded once and replayed on other inputs, with eager work between the replays."""
    torch = torch_mod()
    blocks, weights, gates, r, y = trunk(wl.BF16, 2, gate_rows=11, sigmoid=True)
    head = TrainingHead(ROWS, D, V, r.dtype)
    g = torch.Generator(device="cuda").manual_seed(4)
    w, target = torch.randn(V, D, generator=g, device="cuda").to(r.dtype), torch.randint(0, V, (ROWS,), generator=g, device="cuda")
    g_logp = torch.full((ROWS,), -1.0 / ROWS, device="cuda")
    update = blk.OrthogonalUpdate(2, HIDDEN, D, r.dtype, momentum=0.0)

    def step():
        a, b = r, y
        for m, p, gt in zip(blocks, weights, gates):
            a, b = m.forward(a, b, p, gt)
        head.forward(a, None, None, w, target)
        d, dy = head.backward(g_logp)[0], None
        for m in reversed(blocks):
            d, dy = m.backward(d, dy)
        return d, dy, update.step([m.grads["w1"] for m in blocks])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    for i in range(4):
        r.copy_(torch.randn(ROWS, D, generator=g, device="cuda"))
        y.copy_(torch.randn(ROWS, D, generator=g, device="cuda"))
        eager = [t.clone() for t in step()]
        for t in recorded:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(recorded, eager):
            assert torch.equal(got, want), i


def test_two_chains_on_two_streams():
    torch = torch_mod()
    sets = [trunk(wl.F16, 2, seed=s, gate_rows=3) for s in (1, 2)]
    dr = torch.randn(ROWS, D, device="cuda").half()
    alone = [[t.clone() for t in run(*s, dr)] for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    together = [None, None]
    for _ in range(5):
        for i, s in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                together[i] = run(*s, dr)
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        for x, z in zip(a, b):
            assert torch.equal(x, z)


def test_the_update_against_its_definition():
    torch = torch_mod()
    from oracle import rows_oracle as ro
    from test_gpu_orthogonal import STEP
    from test_gpu_orthogonal import bound as steps_bound

    u = blk.OrthogonalUpdate(3, 24, 40, torch.float32, momentum=0.9)
    g = torch.Generator(device="cuda").manual_seed(5)
    m = np.zeros((3, 24, 40))
    for _ in range(3):
        grads = [torch.randn(24, 40, generator=g, device="cuda") for _ in range(3)]
        got = u.step(grads).double().cpu().numpy()
        gn = np.stack([t.double().cpu().numpy() for t in grads])
        m = 0.9 * m + gn
        for i in range(3):
            want = ro.newton_schulz(gn[i] + 0.9 * m[i], 5, STEP, 1e-7)
            # (the momentum's own roundings, three a step, move the matrix before its steps)
            assert np.linalg.norm(got[i] - want) <= (steps_bound(wl.F32, 24, 40, 5, STEP) + 9 * EPS32 * 3.4445 ** 5) * np.linalg.norm(want)


def test_what_does_not_fit_is_refused():
    torch = torch_mod()
    blocks, weights, gates, r, y = trunk(wl.F16, 1, gate_rows=3)
    b, p, gt = blocks[0], weights[0], gates[0]
    for bad in (r[:-1], r.float(), r.cpu(), torch.empty(D, ROWS, dtype=r.dtype, device="cuda").t()):
        with pytest.raises(ValueError):
            b.forward(bad, y, p, gt)
        with pytest.raises(ValueError):
            b.forward(r, bad, p, gt)
    with pytest.raises(ValueError):
        b.forward(r, y, {k: v for k, v in p.items() if k != "b1"}, gt)
    with pytest.raises(ValueError):
        b.forward(r, y, dict(p, w1=p["w2"]), gt)
    with pytest.raises(ValueError):
        b.forward(r, y, p)
    with pytest.raises(ValueError):
        b.forward(r, y, p, gt[:-1])
    with pytest.raises(RuntimeError):
        b.backward(r)
    b.forward(r, y, p, gt)
    with pytest.raises(ValueError):
        b.backward(r, y)  # a last block has no y
    b.backward(r)
    with pytest.raises(RuntimeError):
        b.backward(r)
    with pytest.raises(ValueError):
        blk.TrainingBlock(4, 8, 8, torch.float16, device="cpu")
    u = blk.OrthogonalUpdate(2, 4, 6, torch.float32)
    ok = torch.ones(4, 6, device="cuda")
    for bad in ([ok], [ok, ok.t()], [ok, ok.cpu()], [ok, ok.int()]):
        with pytest.raises(ValueError):
            u.step(bad)


def test_the_command_runs():
    lines = []
    first, last = blk.demo(images=3, pixels=10, D=32, hidden=48, classes=7, steps=3, log=lines.append)
    assert len(lines) == 2 and np.isfinite([first, last]).all()


def test_a_block_without_rows_has_gradients_of_zeros():
    torch = torch_mod()
    b = blk.TrainingBlock(0, D, HIDDEN, torch.bfloat16, gate_rows=3, sigmoid=True)
    weights = {k: torch.ones(*s, dtype=b.dtype if k in blk.WEIGHTS else torch.float32, device="cuda") for k, s in b.shapes.items()}
    for g in b.grads.values():
        g.fill_(7.0)
    none = torch.empty(0, D, dtype=b.dtype, device="cuda")
    b.forward(none, none, weights, none)
    b.backward(none, none)
    assert all(not bool(g.any()) for g in b.grads.values())


def test_fp16_directions_of_gradients_outside_the_types_range():
    torch = torch_mod()
    from oracle import rows_oracle as ro
    from test_gpu_orthogonal import STEP
    from test_gpu_orthogonal import bound as steps_bound

    u = blk.OrthogonalUpdate(2, 24, 40, torch.float16, momentum=0.5, nesterov=False, eps=0.0)
    grads = torch.randn(2, 24, 40, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda") * torch.tensor([1e-9, 1e6], device="cuda").view(2, 1, 1)
    got = u.step(list(grads)).double().cpu().numpy()
    assert u.direction.dtype == torch.float16
    for i in range(2):
        want = ro.newton_schulz(grads[i].double().cpu().numpy(), 5, STEP, 0.0)
        assert np.linalg.norm(got[i] - want) <= steps_bound(wl.F16, 24, 40, 5, STEP) * np.linalg.norm(want)
