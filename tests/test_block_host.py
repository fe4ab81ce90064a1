"""The operators of a block of rows without a GPU: refusals of every entry point, empty calls, and the oracle against differences."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B

P = 1 << 20  # an aligned address that is never read: every call here ends before the first HIP call


def status(call, *args, **kw):
    try:
        call(*args, **kw)
    except B.ConvError as e:
        return e.status
    return B.CONV_OK


def fwd(d, x=P, w=2 * P, bias=P, residual=3 * P, out=4 * P, pre=5 * P, ws=P, n=1 << 40):
    return status(B.linear_fwd, d, x, w, bias, residual, out, pre, ws, n, stream=0)


def bwd(d, x=P, w=2 * P, pre=3 * P, dout=4 * P, dx=5 * P, dw=6 * P, dbias=7 * P, ws=P, n=1 << 40):
    return status(B.linear_bwd, d, x, w, pre, dout, dx, dw, dbias, ws, n, stream=0)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(rows=1 << 31), dict(N=0), dict(K=0), dict(N=1 << 24), dict(K=1 << 24), dict(ldx=15), dict(ldw=15), dict(ldr=7),
                                    dict(ldo=7), dict(flags=2), dict(flags=B.CONV_FLAG_RELU | B.LINEAR_FLAG_GELU), dict(flags=0x300), dict(ldx=1 << 62), dict(ldo=1 << 61)])
def test_linear_descriptors_that_are_refused(change):
    d = B.make_linear_desc(4, 8, 16, B.CONV_BF16)
    for k, v in change.items():
        setattr(d, k, v)
    if change == dict(N=1 << 24):
        d.ldr = d.ldo = 1 << 24
    if change == dict(K=1 << 24):
        d.ldx = d.ldw = 1 << 24
    assert fwd(d) == B.CONV_EINVAL and bwd(d) == B.CONV_EINVAL
    assert B.linear_workspace_bytes(d) == 0 and B.linear_bwd_workspace_bytes(d) == 0
    with pytest.raises(B.ConvError):
        B.linear_form(d)


def test_linear_types_and_activations_that_are_refused():
    d = B.make_linear_desc(4, 8, 16)
    d.dtype = 3
    assert fwd(d) == B.CONV_EDTYPE and bwd(d) == B.CONV_EDTYPE
    with pytest.raises(KeyError):
        B.make_linear_desc(4, 8, 16, act="tanh")


def test_linear_pointers_that_are_refused():
    d = B.make_linear_desc(4, 8, 16, B.CONV_BF16)
    for name in ("x", "w", "out"):
        assert fwd(d, **{name: None}) == B.CONV_EINVAL
    for name in ("x", "w", "out", "residual", "pre"):
        assert fwd(d, **{name: 9 * P + 1}) == B.CONV_EINVAL
    assert fwd(d, bias=P + 2) == B.CONV_EINVAL
    assert fwd(d, out=P) == B.CONV_EINVAL and fwd(d, out=2 * P) == B.CONV_EINVAL and fwd(d, pre=4 * P) == B.CONV_EINVAL
    assert fwd(d, pre=P) == B.CONV_EINVAL and fwd(d, pre=2 * P) == B.CONV_EINVAL and fwd(d, pre=3 * P) == B.CONV_EINVAL
    d.ldr = 9
    assert fwd(d, residual=4 * P) == B.CONV_EINVAL  # over the residual, other strides
    assert B.lib().linear_fwd(None, P, P, P, P, P, P, P, 0, None) == B.CONV_EINVAL
    d = B.make_linear_desc(4, 8, 16, B.CONV_F32)
    assert fwd(d, x=P + 2) == B.CONV_EINVAL


def test_linear_bwd_pointers_that_are_refused():
    d = B.make_linear_desc(4, 8, 16, B.CONV_F16, act="gelu")
    assert bwd(d, dx=None, dw=None, dbias=None) == B.CONV_EINVAL  # nothing asked for
    for name in ("x", "w", "pre", "dout"):
        assert bwd(d, **{name: None}) == B.CONV_EINVAL
    for name in ("x", "w", "pre", "dout", "dx", "dw"):
        assert bwd(d, **{name: 9 * P + 1}) == B.CONV_EINVAL
    assert bwd(d, dbias=P + 2) == B.CONV_EINVAL
    for taken in (P, 2 * P, 3 * P, 4 * P):
        assert bwd(d, dx=taken) == B.CONV_EINVAL and bwd(d, dw=taken) == B.CONV_EINVAL
    assert bwd(d, dx=6 * P) == B.CONV_EINVAL
    assert B.lib().linear_bwd(None, P, P, P, P, P, P, P, P, 0, None) == B.CONV_EINVAL


def test_linear_workspaces_that_are_refused():
    d = B.make_linear_desc(8192, 8192, 4096)
    for call, need in ((fwd, B.linear_workspace_bytes(d)), (bwd, B.linear_bwd_workspace_bytes(d))):
        assert need > 0
        assert call(d, ws=None, n=need) == B.CONV_EWORKSPACE
        assert call(d, n=need - 1) == B.CONV_EWORKSPACE
        assert call(d, ws=P + 8, n=need) == B.CONV_EINVAL


def test_linear_without_rows():
    d = B.make_linear_desc(0, 8, 16)
    assert B.linear_workspace_bytes(d) == 0 and B.linear_bwd_workspace_bytes(d) == 0
    assert fwd(d, None, None, None, None, None, None, None, 0) == B.CONV_OK
    assert B.linear_form(d) == ""


def test_linear_forms():
    names = {B.linear_form(B.make_linear_desc(r, n, k, B.CONV_BF16), 0, 0) for r, n, k in ((1, 4096, 4096), (2048, 2048, 2048), (8192, 8192, 8192), (1024, 1024, 1024))}
    assert names >= {"rows16", "tile256x256"} and len(names) >= 3
    assert B.linear_form(B.make_linear_desc(2048, 1001, 2048, B.CONV_BF16), 0, 2).endswith("_any")
    assert B.linear_form(B.make_linear_desc(2048, 2048, 2048, B.CONV_F32)).startswith("planes_")
    assert "_split" in B.linear_form(B.make_linear_desc(65536, 256, 256, B.CONV_BF16), which=2)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_oracle_gradients_against_differences(act):
    rng = np.random.default_rng(3)
    x, w, b, g = rng.normal(size=(3, 5)), rng.normal(size=(4, 5)), rng.normal(size=4), rng.normal(size=(3, 4))

    def value(x, w, b):
        return float((g * ro.linear(x, w, b, None, act)[0]).sum())

    dx, dw, db = ro.linear_bwd(x, w, ro.linear(x, w, b, None, act)[1], g, act)
    h = 1e-6
    for t, d, at in ((x, dx, 0), (w, dw, 1), (b, db, 2)):
        for i in np.ndindex(t.shape):
            args = [x.copy(), w.copy(), b.copy()]
            args[at][i] += h
            up = value(*args)
            args[at][i] -= 2 * h
            assert abs((up - value(*args)) / (2 * h) - d[i]) < 1e-6
