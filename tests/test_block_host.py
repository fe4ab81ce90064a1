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
    assert fwd(d, bias=4 * P) == B.CONV_EINVAL
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
    assert bwd(d, dx=6 * P) == B.CONV_EINVAL and bwd(d, dbias=6 * P) == B.CONV_EINVAL and bwd(d, dbias=4 * P) == B.CONV_EINVAL
    assert B.lib().linear_bwd(None, P, P, P, P, P, P, P, P, 0, None) == B.CONV_EINVAL


def test_linear_workspaces_that_are_refused():
    d = B.make_linear_desc(256, 256, 1 << 16, B.CONV_BF16)  # a long reduction for few tiles, shared by workgroups
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
    assert B.linear_form(B.make_linear_desc(2048, 2048, 2048, B.CONV_F32)).startswith("split_")
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


# ---- the norms around a block ------------------------------------------------------------------------------------------


def nfwd(d, r=P, h=2 * P, gate=3 * P, gamma_h=P, beta_h=P, scale=P, gamma=P, beta=P, r_out=4 * P, y=5 * P, stats=6 * P):
    return status(B.residual_norm_fwd, d, r, h, gate, gamma_h, beta_h, scale, gamma, beta, r_out, y, stats, stream=0)


def nbwd(d, r_out=P, h=2 * P, gate=3 * P, gamma_h=P + 64, beta_h=P + 64, scale=P + 64, gamma=P + 64, stats=4 * P, dr_out=5 * P, dy=6 * P, dr=7 * P, dh=8 * P, dgate=9 * P,
         dgamma_h=10 * P, dbeta_h=11 * P, dscale=12 * P, dgamma=13 * P, dbeta=14 * P, ws=P, n=1 << 40):
    return status(B.residual_norm_bwd, d, r_out, h, gate, gamma_h, beta_h, scale, gamma, stats, dr_out, dy, dr, dh, dgate, dgamma_h, dbeta_h, dscale, dgamma, dbeta,
                  ws, n, stream=0)


@pytest.mark.parametrize("change", [dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=1 << 27), dict(ldr=7), dict(ldh=7), dict(ldy=7), dict(ldg=7), dict(gate_rows=-1),
                                    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(flags=8), dict(ldr=1 << 62), dict(ldg=1 << 62)])
def test_residual_norm_descriptors_that_are_refused(change):
    d = B.make_residual_norm_desc(4, 8, B.CONV_BF16, gate_rows=2)
    for k, v in change.items():
        setattr(d, k, v)
    if change == dict(cols=1 << 27):
        d.ldr = d.ldh = d.ldy = d.ldg = 1 << 27
    assert nfwd(d) == B.CONV_EINVAL and nbwd(d) == B.CONV_EINVAL
    assert B.residual_norm_bwd_workspace_bytes(d) == 0


def test_residual_norm_pointers_that_are_refused():
    d = B.make_residual_norm_desc(4, 8, B.CONV_BF16, gate_rows=2)
    for name in ("r", "h", "r_out", "gate"):
        assert nfwd(d, **{name: None}) == B.CONV_EINVAL
    for name in ("r", "h", "gate", "r_out", "y", "gamma_h", "beta_h", "scale", "gamma", "beta", "stats"):
        assert nfwd(d, **{name: 17 * P + 1}) == B.CONV_EINVAL
    assert nfwd(d, stats=17 * P + 4) == B.CONV_EINVAL                       # its rows are read four floats at a time
    assert nfwd(d, r_out=2 * P) == B.CONV_EINVAL and nfwd(d, r_out=3 * P) == B.CONV_EINVAL
    assert nfwd(d, y=P) == B.CONV_EINVAL and nfwd(d, y=2 * P) == B.CONV_EINVAL and nfwd(d, y=4 * P) == B.CONV_EINVAL
    assert nfwd(d, stats=P) == B.CONV_EINVAL
    d.dtype = 3
    assert nfwd(d) == B.CONV_EDTYPE and nbwd(d) == B.CONV_EDTYPE
    d = B.make_residual_norm_desc(4, 8, post=False)
    assert nfwd(d, gate=None) == B.CONV_EINVAL                              # a norm's vectors without the norm
    assert nfwd(d, gamma_h=None, beta_h=None) == B.CONV_EINVAL              # a gate without rows that share it
    assert B.lib().residual_norm_fwd(None, *[P] * 12) == B.CONV_EINVAL


def test_residual_norm_bwd_pointers_that_are_refused():
    d = B.make_residual_norm_desc(4, 8, B.CONV_BF16, gate_rows=2)
    outs = ("dr", "dh", "dgate", "dgamma_h", "dbeta_h", "dscale", "dgamma", "dbeta")
    assert nbwd(d, **{k: None for k in outs}) == B.CONV_EINVAL              # nothing asked for
    assert nbwd(d, dr_out=None, dy=None) == B.CONV_EINVAL                   # nothing to go by
    for name in ("r_out", "h", "gate", "stats"):
        assert nbwd(d, **{name: None}) == B.CONV_EINVAL
    for name in outs + ("r_out", "h", "gate", "dr_out", "dy", "gamma_h", "scale", "stats"):
        assert nbwd(d, **{name: 17 * P + 1}) == B.CONV_EINVAL
    for name in outs:
        for taken in (P, 2 * P, 3 * P, 4 * P, 5 * P, 6 * P, (8 if name == "dr" else 7) * P):
            assert nbwd(d, **{name: taken}) == B.CONV_EINVAL
    need = B.residual_norm_bwd_workspace_bytes(d)
    assert need > 0
    assert nbwd(d, n=need - 1) == B.CONV_EWORKSPACE and nbwd(d, ws=None, n=need) == B.CONV_EWORKSPACE
    assert nbwd(d, ws=P + 8, n=need) == B.CONV_EINVAL
    d = B.make_residual_norm_desc(4, 8, post=False)
    free = dict(gate=None, gamma_h=None, beta_h=None)
    assert nbwd(d, **free, dgate=None) == B.CONV_EINVAL                     # gradients of vectors that are not there
    assert nbwd(d, **free, dgamma_h=None, dbeta_h=None) == B.CONV_EINVAL    # ... and of gates
    assert B.lib().residual_norm_bwd(None, *[P] * 19, P, 0, None) == B.CONV_EINVAL


def test_residual_norm_without_rows():
    d = B.make_residual_norm_desc(0, 8)
    assert nfwd(d, None, None, None, r_out=None, y=None, stats=None) == B.CONV_OK


@pytest.mark.parametrize("post,rms,gate_rows,sigmoid", [(True, False, 0, False), (True, True, 2, True), (False, False, 1, False), (True, False, 3, True)])
def test_oracle_gradients_of_the_norms_against_differences(post, rms, gate_rows, sigmoid):
    rng = np.random.default_rng(5)
    t = dict(r=rng.normal(size=(5, 6)), h=rng.normal(size=(5, 6)), gate=rng.normal(size=(-(-5 // gate_rows), 6)) if gate_rows else None)
    v = {k: rng.normal(size=6) for k in ("gamma_h", "beta_h", "scale", "gamma", "beta")}
    if not post:
        v["gamma_h"] = v["beta_h"] = None
    gr, gy = rng.normal(size=(5, 6)), rng.normal(size=(5, 6))

    def value(a):
        x, y, _, _ = ro.residual_norm(a["r"], a["h"], a["gate"], gate_rows, sigmoid, a["gamma_h"], a["beta_h"], a["scale"], a["gamma"], a["beta"], post, rms, 1e-3)
        return float((gr * x + gy * y).sum())

    a = {**t, **v}
    x, _, st, _ = ro.residual_norm(a["r"], a["h"], a["gate"], gate_rows, sigmoid, a["gamma_h"], a["beta_h"], a["scale"], a["gamma"], a["beta"], post, rms, 1e-3)
    got = ro.residual_norm_bwd(x, a["h"], a["gate"], gate_rows, sigmoid, a["gamma_h"], a["beta_h"], a["scale"], a["gamma"], st, gr, gy, post, rms)
    e = 1e-6
    for k in a:
        if a[k] is None:
            continue
        for i in np.ndindex(a[k].shape):
            moved = [value({**a, k: a[k] + s * e * (np.indices(a[k].shape) == np.array(i).reshape(-1, *[1] * a[k].ndim)).all(0)}) for s in (1, -1)]
            assert abs((moved[0] - moved[1]) / (2 * e) - got["d" + k][i]) < 1e-6, (k, i)


# ---- Newton-Schulz steps -----------------------------------------------------------------------------------------------


def ns(d, x=P, out=2 * P, ws=P, n=1 << 62):
    return status(B.orthogonalize, d, x, out, ws, n, stream=0)


@pytest.mark.parametrize("change", [dict(batch=-1), dict(batch=1 << 31), dict(rows=0), dict(cols=0), dict(rows=(1 << 20) + 1), dict(steps=0), dict(steps=101), dict(ldx=7), dict(ldo=7),
                                    dict(stride_x=-1), dict(stride_o=31), dict(a=float("nan")), dict(b=float("inf")), dict(c=float("nan")), dict(eps=-1.0), dict(eps=float("nan")),
                                    dict(stride_o=1 << 62), dict(rows=1 << 18, cols=1 << 18, ldx=1 << 18, ldo=1 << 18, stride_o=1 << 36)])
def test_orthogonal_descriptors_that_are_refused(change):
    d = B.make_orthogonal_desc(4, 8, B.CONV_BF16, batch=2)
    for k, v in change.items():
        setattr(d, k, v)
    assert ns(d) == B.CONV_EINVAL and B.orthogonalize_workspace_bytes(d) == 0


def test_orthogonal_arguments_that_are_refused():
    d = B.make_orthogonal_desc(4, 8, B.CONV_F32, batch=2)
    need = B.orthogonalize_workspace_bytes(d)
    assert need > 0
    assert ns(d, x=None) == B.CONV_EINVAL and ns(d, out=None) == B.CONV_EINVAL and ns(d, x=P + 2) == B.CONV_EINVAL and ns(d, out=P + 1) == B.CONV_EINVAL
    assert ns(d, n=need - 1) == B.CONV_EWORKSPACE and ns(d, ws=None) == B.CONV_EWORKSPACE and ns(d, ws=P + 8) == B.CONV_EINVAL
    d.ldx, d.stride_x = 9, 36
    assert ns(d, out=P) == B.CONV_EINVAL                  # in place with other strides
    d.dtype = 3
    assert ns(d) == B.CONV_EDTYPE
    assert ns(B.make_orthogonal_desc(4, 8, batch=0), None, None, None, 0) == B.CONV_OK
    assert B.lib().orthogonalize(None, P, P, P, 0, None) == B.CONV_EINVAL
    assert B.lib().orthogonalize_workspace_bytes(None) == 0


def test_oracle_of_the_steps_against_singular_values():
    x = np.random.default_rng(1).normal(size=(6, 9))
    u, s, v = np.linalg.svd(x / np.linalg.norm(x), full_matrices=False)
    for _ in range(3):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    assert np.allclose(ro.newton_schulz(x, 3, (3.4445, -4.7750, 2.0315), 0.0), u * s @ v, atol=1e-12)


@pytest.mark.parametrize("dtype", [B.CONV_F32, B.CONV_F16, B.CONV_BF16])
@pytest.mark.parametrize("rows,cols", [(1, 40), (100, 64), (4096, 1000), (300, 9000)])
def test_a_gate_for_more_rows_than_there_are_is_one_for_all(rows, cols, dtype):
    """Rows are shared out among workgroups by what there is of them, and so is the room for their sums."""
    need = [B.residual_norm_bwd_workspace_bytes(B.make_residual_norm_desc(rows, cols, dtype, gate_rows=n)) for n in (max(2, rows), 2 * rows + 1, (1 << 31) - 1)]
    assert need[0] == need[1] == need[2]


def test_fp32_rows_take_the_faster_form():
    """fp32 matrix instructions are slow enough to count: many rows over few outputs go through tiles, few rows and very few outputs do not."""
    form = lambda r, n, k: B.linear_form(B.make_linear_desc(r, n, k, B.CONV_F32), 0, 0)  # noqa: E731
    for many in ((114048, 45, 576), (18000, 160, 576), (1744, 62, 3476)):
        assert form(*many).startswith("split_tile"), many
    assert form(24, 46704, 6752).startswith("rows32") and form(17, 4096, 4096) == "rows32"
    for few in ((100000, 16, 256), (4000, 40, 300), (20000, 31, 1000), (128, 4096, 512), (200, 1000, 1000)):
        assert form(*few).startswith("rows64"), few


def test_fp32_gradients_take_the_faster_form():
    """Lone small tiles of operands that lie across the reduction are slower than larger ones that share it; several of them on a CU are faster."""
    form = lambda r, n, k, which: B.linear_form(B.make_linear_desc(r, n, k, B.CONV_F32), 0, 0, which)  # noqa: E731
    for size, which in (((600, 1000, 1000), 1), ((1300, 1111, 640), 2), ((1000, 300, 2000), 2)):
        assert form(*size, which).startswith("split_tile128x128_split"), size
    for size, which in (((600, 1000, 1000), 2), ((300, 700, 3000), 1), ((400, 3000, 400), 2), ((300, 300, 300), 1), ((1024, 1024, 1024), 0)):
        assert form(*size, which) == "split_tile64x64", size


def test_few_fp32_rows_over_many_outputs_take_more_of_them_a_workgroup():
    """x is read again for every workgroup's outputs, which takes longer than the weights."""
    form = lambda r, n, k, at: B.linear_form(B.make_linear_desc(r, n, k, B.CONV_F32), at, at)  # noqa: E731
    assert form(24, 46704, 6752, 0) == "rows32x64" and form(64, 16000, 4096, 0) == "rows64x64"
    assert form(16, 16001, 4099, 4) == "rows16x32_any" and form(30, 16001, 4099, 4) == "rows32x32_any"
    assert form(1, 16000, 4096, 0) == "rows16" and form(20, 8192, 1024, 0) == "rows32" and form(5, 4099, 999, 4) == "rows16_any"
