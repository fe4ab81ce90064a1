"""The training block and the orthogonal update without a GPU: what they hand to the library, and what they refuse before anything is launched.

The binding's launching functions are replaced by ones that write down their arguments, so tensors can lie in host memory; descriptors and workspace
sizes are the library's own."""
import pytest
import torch

from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import block as blk

LAUNCHES = ("linear_fwd", "linear_bwd", "residual_norm_fwd", "residual_norm_bwd", "orthogonalize")
ROWS, D, HIDDEN = 12, 16, 40


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(blk, "GPU", "cpu", raising=False)
    for name in LAUNCHES:
        monkeypatch.setattr(B, name, lambda *args, name=name: made.append((name, args)))
    return made


def block(dtype=torch.bfloat16, **kw):
    return blk.TrainingBlock(ROWS, D, HIDDEN, dtype, device="cpu", **kw)


def weights_of(b):
    return {k: torch.ones(*s, dtype=b.dtype if k in blk.WEIGHTS else torch.float32) for k, s in b.shapes.items()}


def rows_of(b, n=1):
    return [torch.zeros(ROWS, D, dtype=b.dtype) for _ in range(n)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", [dict(), dict(post=False, rms=True), dict(last=True), dict(gate_rows=5, sigmoid=True, act="silu")])
def test_what_a_block_hands_on(calls, kind, dtype):
    b = block(dtype, **kind)
    p, (r, y) = weights_of(b), rows_of(b, 2)
    gate = torch.zeros(3, D, dtype=dtype) if "gate_rows" in kind else None
    out = b.forward(r, y, p, gate)
    assert out == (b.r_out, b.y) and (b.y is None) == ("last" in kind)
    assert [n for n, _ in calls] == ["linear_fwd", "linear_fwd", "residual_norm_fwd"]
    first, second, norm = (a for _, a in calls)
    assert first[1] is y and first[2] is p["w1"] and first[3] is p["b1"] and first[4] is None and first[5] is b.a and first[6] is b.pre
    assert second[1] is b.a and second[2] is p["w2"] and second[5] is b.h and second[6] is None
    assert norm[1] is r and norm[2] is b.h and norm[3] is gate and norm[9] is b.r_out and norm[10] is b.y
    assert (norm[4] is None) == (kind.get("post") is False)
    del calls[:]
    (dr_out,) = rows_of(b)
    assert b.backward(dr_out) == (b.dr, b.dy)
    assert [n for n, _ in calls] == ["residual_norm_bwd", "linear_bwd", "linear_bwd"]
    for name, a in calls:  # one workspace, large enough for every call
        need = (B.residual_norm_bwd_workspace_bytes if name == "residual_norm_bwd" else B.linear_bwd_workspace_bytes)(a[0])
        assert a[-3] is b.ws and a[-2] == b.ws.numel() >= need
    assert set(b.grads) == set(b.shapes) and all(tuple(b.grads[k].shape) == s for k, s in b.shapes.items())
    with pytest.raises(RuntimeError):
        b.backward(dr_out)  # a second time


def test_rows_that_are_refused(calls):
    b = block()
    p, (r, y) = weights_of(b), rows_of(b, 2)
    for bad in (torch.zeros(ROWS, D), torch.zeros(ROWS - 1, D, dtype=b.dtype), torch.zeros(ROWS, 2 * D, dtype=b.dtype)[:, ::2], torch.zeros(D, ROWS, dtype=b.dtype).t(),
                torch.zeros(ROWS, D, dtype=b.dtype, device="meta"), torch.zeros(ROWS, D, 1, dtype=b.dtype)):
        with pytest.raises(ValueError):
            b.forward(bad, y, p)
        with pytest.raises(ValueError):
            b.forward(r, bad, p)
    with pytest.raises(ValueError):
        b.forward(r, b.y, p)  # its own result: replaced before the gradient reads it
    assert not calls
    b.forward(r, y, p)
    with pytest.raises(ValueError):
        b.backward(torch.zeros(ROWS, D))
    with pytest.raises(ValueError):
        b.backward(*rows_of(b), torch.zeros(ROWS, D))
    b.backward(*rows_of(b, 2))  # a refused call does not use the forward pass up
    assert len(calls) == 6


def test_weights_and_gates_that_are_refused(calls):
    b = block(gate_rows=4)
    r, y = rows_of(b, 2)
    gate = torch.zeros(3, D, dtype=b.dtype)
    for k in b.shapes:
        p = weights_of(b)
        for bad in (p[k].double(), p[k][..., :-1], torch.ones(*(2 * s for s in p[k].shape), dtype=p[k].dtype)[tuple(slice(None, None, 2) for _ in p[k].shape)]):
            with pytest.raises(ValueError):
                b.forward(r, y, {**p, k: bad}, gate)
        del p[k]
        with pytest.raises(ValueError):
            b.forward(r, y, p, gate)
    p = weights_of(b)
    for bad in (None, gate[:2], gate.float(), torch.zeros(4, D, dtype=b.dtype)):
        with pytest.raises(ValueError):
            b.forward(r, y, p, bad)
    with pytest.raises(ValueError):
        block().forward(r, y, weights_of(block()), gate)
    with pytest.raises(ValueError):
        b.forward(r, y, {**p, "other": p["b1"]}, gate)
    with pytest.raises(RuntimeError):
        b.backward(*rows_of(b))  # no forward pass was accepted
    last = block(last=True)
    last.forward(r, y, weights_of(last))
    with pytest.raises(ValueError):
        last.backward(*rows_of(last, 2))
    assert len(calls) == 3


def test_places_and_types_that_are_refused():
    with pytest.raises(ValueError):
        blk.TrainingBlock(4, 8, 16, torch.float32, device="cpu")
    with pytest.raises(ValueError):
        blk.OrthogonalUpdate(2, 8, 16, torch.float32, device="cpu")


@pytest.mark.parametrize("nesterov", [True, False])
def test_momentum_of_the_update(calls, nesterov):
    u = blk.OrthogonalUpdate(2, 3, 5, torch.float32, momentum=0.5, nesterov=nesterov, device="cpu")
    g = torch.Generator().manual_seed(1)
    total = torch.zeros(2, 3, 5)
    for step in range(3):
        grads = [torch.randn(3, 5, generator=g) for _ in range(2)]
        assert u.step(grads) is u.direction
        now = torch.stack(grads)
        total = 0.5 * total + now
        assert torch.allclose(u.sum, total) and torch.allclose(u.direction, 0.5 * total + now if nesterov else total)
        name, a = calls[step]
        assert name == "orthogonalize" and a[1] is a[2] is u.direction and a[4] == u.ws.numel() >= B.orthogonalize_workspace_bytes(a[0])
    before = u.sum.clone()
    for bad in ([grads[0]], [grads[0], grads[1].t()], [grads[0], grads[1].int()], [grads[0], grads[1].to("meta")]):
        with pytest.raises(ValueError):
            u.step(bad)
    assert torch.equal(u.sum, before) and len(calls) == 3


def test_a_block_without_rows(calls):
    """All tensors of no rows have the address zero, the block's own result too."""
    b = blk.TrainingBlock(0, D, HIDDEN, torch.float32, gate_rows=3, device="cpu")
    r, y = torch.zeros(0, D), torch.zeros(0, D)
    assert b.forward(r, y, weights_of(b), torch.zeros(0, D)) == (b.r_out, b.y)
    assert b.backward(torch.zeros(0, D), torch.zeros(0, D)) == (b.dr, b.dy)
    assert len(calls) == 6


def test_a_call_that_the_library_refuses_does_not_use_the_forward_pass_up(calls, monkeypatch):
    """As when a gradient is handed in where the block writes one."""
    b = block()
    b.forward(*rows_of(b, 2), weights_of(b))

    def refuse(*args):
        raise B.ConvError(B.CONV_EINVAL, "residual_norm_bwd")

    taken = B.residual_norm_bwd
    monkeypatch.setattr(B, "residual_norm_bwd", refuse)
    with pytest.raises(B.ConvError):
        b.backward(b.dr)
    monkeypatch.setattr(B, "residual_norm_bwd", taken)
    assert b.backward(*rows_of(b, 2)) == (b.dr, b.dy)
    with pytest.raises(RuntimeError):
        b.backward(*rows_of(b, 2))


def test_the_momentum_may_leave_the_range_of_fp16(calls):
    """Gradients of 1e-9 vanish in fp16, and twenty times one of 6e4, as the momentum adds them up, is an infinity there."""
    u = blk.OrthogonalUpdate(2, 3, 5, torch.float16, device="cpu")
    small, large = torch.full((3, 5), 1e-9), torch.full((3, 5), 6e4, dtype=torch.float16)
    for _ in range(30):
        out = u.step([small, large])
    assert out.dtype == torch.float16 and out is u.direction
    handed = calls[-1][1][1]
    assert calls[-1][1][2] is handed and bool(torch.isfinite(handed).all()) and bool((handed != 0).all())
    assert calls[-1][1][4] >= B.orthogonalize_workspace_bytes(calls[-1][1][0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_the_direction_has_the_updates_type(calls, dtype):
    u = blk.OrthogonalUpdate(1, 3, 5, dtype, momentum=0.0, device="cpu")
    g = torch.arange(15.0).view(3, 5)
    assert torch.equal(u.step([g]), g[None].to(dtype)) and u.direction.dtype == dtype  # (the steps, which are not made here, work in place)


def test_another_current_device_is_refused(calls, monkeypatch):
    """Kernels are launched on the current device, which another one's memory is not for."""
    current = [0]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    blk._current(torch, torch.device("cuda:0"))
    with pytest.raises(ValueError):
        blk._current(torch, torch.device("cuda:1"))
    current[0] = 1
    blk._current(torch, torch.device("cuda:1"))

    def other(torch, device):
        raise ValueError("another device")

    b, u = block(), blk.OrthogonalUpdate(1, 3, 5, torch.float32, device="cpu")
    b.forward(*rows_of(b, 2), weights_of(b))
    del calls[:]
    before = u.sum.clone()
    monkeypatch.setattr(blk, "_current", other)
    for call in (lambda: b.forward(*rows_of(b, 2), weights_of(b)), lambda: b.backward(*rows_of(b, 2)), lambda: u.step([torch.ones(3, 5)])):
        with pytest.raises(ValueError):
            call()
    assert not calls and torch.equal(u.sum, before)
