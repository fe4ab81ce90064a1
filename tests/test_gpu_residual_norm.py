"""The norms around a block on the GPU, forward and backward, against 64 bits.

Bounds (first order, one rounding is EPS32): a row's sum is formed by chains of at most 16 elements a lane and ten joins (rows that no registers hold: cols / 1024 and
ten), so c = 32 + cols / 1024 roundings of the magnitudes it adds up; the sums over the rows by at most as many roundings as rows and ten; a
sigmoid is off by 6 + |g| roundings.  Errors are carried along by the slopes of what follows them, and each result rounded once to its type."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod
from rows_util import EPS32, ROUND, TINY, Rows, assert_close, nan_vec, stored, torch_type, vec

pytestmark = pytest.mark.gpu

DTYPES = [wl.F32, wl.F16, wl.BF16]
EPS = 1e-5


def one(v):
    return 1.0 if v is None else v.astype(np.float64)


def zero(v):
    return 0.0 if v is None else v.astype(np.float64)


def avg(x):
    return x.mean(1)[:, None]


def make(rows, cols, dtype, post, gate_rows, scale, affine, seed, spread=1.0):
    rng = np.random.default_rng(seed + rows + 7 * cols)
    size = rng.uniform(0.5, 2, (rows, 1))
    t = dict(r=spread * size * rng.normal(size=(rows, cols)) + rng.normal(size=(rows, 1)), h=0.5 * size * rng.normal(size=(rows, cols)) + 0.2,
             dr_out=rng.normal(size=(rows, cols)), dy=rng.normal(size=(rows, cols)))
    t["gate"] = 0.5 + 0.7 * rng.normal(size=(-(-rows // gate_rows), cols)) if gate_rows else None
    t = {k: None if v is None else stored(v, dtype) for k, v in t.items()}
    v = lambda mean: (mean + 0.3 * rng.normal(size=cols)).astype(np.float32)  # noqa: E731
    vectors = dict(gamma_h=v(1) if post and affine else None, beta_h=v(0) if post and affine else None, scale=v(0.5) if scale else None,
                   gamma=v(1) if affine else None, beta=v(0) if affine else None)
    return t, vectors


def check_fwd(rows, cols, dtype, post=True, rms=False, gate_rows=0, sigmoid=False, scale=True, affine=True, y=True, stats=True, pad=0, start=0, seed=0, inplace=False,
              data=None):
    torch = torch_mod()
    tt, nan = torch_type(dtype), float("nan")
    t, v = data or make(rows, cols, dtype, post, gate_rows, scale, affine, seed)
    put = lambda x, extra: Rows(len(x), cols, tt, cols + extra, start, nan).set(x)  # noqa: E731
    R, Hh = put(t["r"], pad), put(t["h"], 2 * pad)
    G = put(t["gate"], 3 * pad) if gate_rows else None
    O, Y = R if inplace else Rows(rows, cols, tt, cols + pad, start, 7.0), Rows(rows, cols, tt, cols + 4 * pad, start, 5.0)
    S = torch.full((rows, 4), nan, device="cuda")
    d = B.make_residual_norm_desc(rows, cols, dtype, EPS, rms, post, gate_rows, sigmoid, R.ld, Hh.ld, G.ld if G else 0, Y.ld)
    dev = {k: None if x is None else vec(x) for k, x in v.items()}
    B.residual_norm_fwd(d, R.ptr, Hh.ptr, G.ptr if G else None, dev["gamma_h"], dev["beta_h"], dev["scale"], dev["gamma"], dev["beta"], O.ptr, Y.ptr if y else None,
                        S if stats else None)
    torch.cuda.synchronize()
    x, ref, st, branch = ro.residual_norm(t["r"], t["h"], t["gate"], gate_rows, sigmoid, *(None if v[k] is None else v[k].astype(np.float64) for k in
                                          ("gamma_h", "beta_h", "scale", "gamma", "beta")), post, rms, EPS)
    c = 32 + cols / 1024
    off = 0.0
    s = one(v["scale"])
    if post:
        hh = (t["h"] - st[:, 0:1]) * st[:, 1:2]
        dm = 0.0 if rms else c * EPS32 * avg(np.abs(t["h"]))
        off = (dm * st[:, 1:2] + np.abs(hh) * (c + 8) * EPS32) * np.abs(s * one(v["gamma_h"])) + 3 * EPS32 * (np.abs(hh * s * one(v["gamma_h"])) + np.abs(s * zero(v["beta_h"])))
    else:
        off = 2 * EPS32 * np.abs(t["h"] * s)
    if gate_rows:
        g = t["gate"][np.arange(rows) // gate_rows]
        off = off * np.abs(1 / (1 + np.exp(-g)) if sigmoid else g) + np.abs(branch) * EPS32 * (6 + np.abs(g))
    off = off + EPS32 * (np.abs(x) + np.abs(branch))
    assert_close(O.host(), x, off + ROUND[dtype] * (np.abs(x) + off) + TINY[dtype], "r_out")
    assert inplace or O.untouched()
    mean, rstd = st[:, 2:3], st[:, 3:4]
    xh = (x - mean) * rstd
    dm = 0.0 if rms else c * EPS32 * avg(np.abs(x)) + avg(off)
    dr = (c + 8) * EPS32 + avg(off * np.abs(xh)) * rstd
    if y:
        tol = np.abs(one(v["gamma"])) * (rstd * (off + dm) + np.abs(xh) * (dr + 2 * EPS32)) + 2 * EPS32 * (np.abs(ref) + np.abs(zero(v["beta"])))
        assert_close(Y.host(), ref, tol + ROUND[dtype] * (np.abs(ref) + tol) + TINY[dtype], "y")
        assert Y.untouched()
    else:
        assert Y.untouched(written=0)
        st[:, 2:] = [0.0, 1.0]
    if stats:
        got = S.cpu().numpy()
        if post:
            assert_close(got[:, 0], st[:, 0], 0.0 if rms else c * EPS32 * np.abs(t["h"]).mean(1) + EPS32 * np.abs(st[:, 0]), "mean of h")
            assert_close(got[:, 1], st[:, 1], (c + 8) * EPS32 * st[:, 1], "rstd of h")
        else:
            assert np.array_equal(got[:, :2], st[:, :2])
        if y:
            assert_close(got[:, 2], st[:, 2], dm[:, 0] + EPS32 * np.abs(st[:, 2]) if not rms else 0.0, "mean")
            assert_close(got[:, 3], st[:, 3], dr[:, 0] * st[:, 3], "rstd")
        else:
            assert np.array_equal(got[:, 2:], st[:, 2:])


OUTPUTS = ("dr", "dh", "dgate", "dgamma_h", "dbeta_h", "dscale", "dgamma", "dbeta")


def check_bwd(rows, cols, dtype, post=True, rms=False, gate_rows=0, sigmoid=False, scale=True, affine=True, dr_out=True, dy=True, pad=0, start=0, seed=0, want=OUTPUTS):
    torch = torch_mod()
    tt, nan = torch_type(dtype), float("nan")
    t, v = make(rows, cols, dtype, post, gate_rows, scale, affine, seed)
    f64 = {k: None if x is None else x.astype(np.float64) for k, x in v.items()}
    x, _, st, _ = ro.residual_norm(t["r"], t["h"], t["gate"], gate_rows, sigmoid, *(f64[k] for k in ("gamma_h", "beta_h", "scale", "gamma", "beta")), post, rms, EPS)
    x, st = stored(x, dtype), st.astype(np.float32).astype(np.float64)
    zeros = np.zeros((rows, cols))
    if not dr_out:
        t["dr_out"] = zeros
    if not dy:
        t["dy"] = zeros
    put = lambda a, extra: Rows(len(a), cols, tt, cols + extra, start, nan).set(a)  # noqa: E731
    out = lambda n, extra: Rows(n, cols, tt, cols + extra, start, 7.0)  # noqa: E731
    X, DRO, Hh, DY = put(x, pad), put(t["dr_out"], pad), put(t["h"], 2 * pad), put(t["dy"], 4 * pad)
    G = put(t["gate"], 3 * pad) if gate_rows else None
    want = [k for k in want if not (k == "dgate" and not gate_rows) and not (k in ("dgamma_h", "dbeta_h") and not post)]
    O = {"dr": out(rows, pad), "dh": out(rows, 2 * pad), "dgate": out(len(t["gate"]), 3 * pad) if gate_rows else None}
    V = {k: nan_vec(cols) for k in OUTPUTS[3:]}
    d = B.make_residual_norm_desc(rows, cols, dtype, EPS, rms, post, gate_rows, sigmoid, X.ld, Hh.ld, G.ld if G else 0, DY.ld)
    need = B.residual_norm_bwd_workspace_bytes(d)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    dev = {k: None if a is None else vec(a) for k, a in v.items()}
    at = lambda k: None if k not in want else O[k].ptr if k in O else V[k]  # noqa: E731
    B.residual_norm_bwd(d, X.ptr, Hh.ptr, G.ptr if G else None, dev["gamma_h"], dev["beta_h"], dev["scale"], dev["gamma"], vec(st), DRO.ptr if dr_out else None,
                        DY.ptr if dy else None, *(at(k) for k in OUTPUTS), ws, need)
    torch.cuda.synchronize()
    ref = ro.residual_norm_bwd(x, t["h"], t["gate"], gate_rows, sigmoid, f64["gamma_h"], f64["beta_h"], f64["scale"], f64["gamma"], st, t["dr_out"], t["dy"], post, rms)
    c = 32 + cols / 1024
    A = np.abs

    def through(g, off, xh, rstd):
        """How far the gradient through a norm is off, where g is off by `off`."""
        e = off + A(xh) * avg(off * A(xh)) + 6 * EPS32 * A(g) + A(xh) * (c + 10) * EPS32 * avg(A(g * xh))
        if not rms:
            e = e + avg(off) + (c + 6) * EPS32 * avg(A(g))
        return rstd * e + 4 * EPS32 * rstd * (A(g) + A(xh) * avg(A(g * xh)) + avg(A(g)))

    s, ga, gb = A(one(v["scale"])), A(one(v["gamma_h"])), A(zero(v["beta_h"]))
    xh, g = (x - st[:, 2:3]) * st[:, 3:4], t["dy"] * one(v["gamma"])
    off = (through(g, EPS32 * A(g), xh, st[:, 3:4]) if dy else 0.0) + 2 * EPS32 * (A(t["dr_out"]) + A(ref["dr"]))
    tol = {"dr": off}
    hh = (t["h"] - st[:, 0:1]) * st[:, 1:2] if post else t["h"]
    size_u = A(hh) * ga + gb
    p, off_p = ref["dr"], off
    if gate_rows:
        row = np.arange(rows) // gate_rows
        gate = t["gate"][row]
        eff = 1 / (1 + np.exp(-gate)) if sigmoid else gate
        slope = 1 / (1 + np.exp(-t["gate"])) * (1 - 1 / (1 + np.exp(-t["gate"]))) if sigmoid else np.ones_like(t["gate"])
        each = off * s * size_u + (gate_rows + 16) * EPS32 * A(p) * s * size_u
        total, mags = np.zeros_like(t["gate"]), np.zeros_like(t["gate"])
        np.add.at(total, row, each)
        np.add.at(mags, row, A(p) * s * size_u)
        tol["dgate"] = total * slope + mags * (slope * 10 + (EPS32 > 0) * slope * 2 * (6 + A(t["gate"])) + (sigmoid * 2.0)) * EPS32
        off_p = off * A(eff) + A(p * eff) * EPS32 * (6 + A(gate))
        p = p * eff
    n = (rows + 12) * EPS32
    tol["dbeta_h"] = s * (off_p.sum(0) + n * A(p).sum(0))
    tol["dgamma_h"] = s * ((off_p * A(hh)).sum(0) + n * A(p * hh).sum(0))
    tol["dscale"] = (off_p * size_u).sum(0) + n * (A(p) * size_u).sum(0)
    tol["dgamma"], tol["dbeta"] = n * A(t["dy"] * xh).sum(0), n * A(t["dy"]).sum(0)
    du, off_du = p * one(v["scale"]) * one(v["gamma_h"]), off_p * s * ga + 3 * EPS32 * A(p) * s * ga
    tol["dh"] = through(du, off_du, hh, st[:, 1:2]) if post else off_du
    for k in OUTPUTS:
        if k in O:
            if k in want:
                assert_close(O[k].host(), ref[k], tol[k] + ROUND[dtype] * (A(ref[k]) + tol[k]) + TINY[dtype], k)
            assert O[k] is None or O[k].untouched(written=None if k in want else 0)
        elif k in want:
            assert_close(V[k].cpu().numpy(), ref[k], tol[k] + EPS32 * A(ref[k]), k)
        else:
            assert bool(torch.isnan(V[k]).all())


SIZES = [(1, 1), (1, 7), (3, 8), (5, 16), (70, 17), (9, 64), (33, 65), (130, 100), (20, 128), (7, 129), (40, 256), (11, 300), (6, 512), (19, 768), (5, 1000), (3, 1024),
         (10, 1537), (2, 2048), (9, 4096), (4, 4097), (3, 5001), (2, 8192), (5, 8193), (3, 9632), (2, 16384), (3, 16390)]
KINDS = [dict(), dict(rms=True, scale=False), dict(post=False), dict(post=False, rms=True, affine=False, scale=False), dict(gate_rows=1, sigmoid=True),
         dict(gate_rows=3), dict(post=False, gate_rows=2, sigmoid=True, scale=False), dict(rms=True, gate_rows=1, affine=False)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_forward(rows, cols, kind):
    check_fwd(rows, cols, DTYPES[(rows + cols + kind) % 3], pad=(rows + kind) % 3, start=cols % 2, seed=kind, **KINDS[kind])


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_backward(rows, cols, kind):
    check_bwd(rows, cols, DTYPES[(rows + cols + kind) % 3], pad=(rows + kind) % 3, start=cols % 2, seed=kind, **KINDS[kind])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,gate_rows", [(3380, 384, 169), (1000, 192, 196), (999, 1000, 49), (2000, 64, 7), (700, 4096, 1), (515, 40, 600), (300, 8200, 100), (5000, 128, 0)])
def test_many_rows(rows, cols, gate_rows, dtype):
    kind = dict(rms=bool(dtype % 2), post=cols % 3 != 0, gate_rows=gate_rows, sigmoid=rows % 2 == 0)
    check_fwd(rows, cols, dtype, **kind)
    check_bwd(rows, cols, dtype, **kind)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [24, 200, 1000, 3000, 20000])
def test_parts_that_are_left_out(cols, dtype):
    for post in (True, False):
        check_fwd(9, cols, dtype, post=post, y=False)
        check_fwd(9, cols, dtype, post=post, stats=False, inplace=True)
        check_fwd(9, cols, dtype, post=post, y=False, gate_rows=4, inplace=True)
        check_bwd(9, cols, dtype, post=post, dr_out=False)
        check_bwd(9, cols, dtype, post=post, dy=False, gate_rows=2)
        for want in (("dr",), ("dh",), ("dgate",), ("dgamma", "dbeta"), ("dgamma_h",), ("dscale",), ("dr", "dh", "dgate")):
            if post or want != ("dgamma_h",):
                check_bwd(9, cols, dtype, post=post, gate_rows=3, want=want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [64, 1000, 4096, 16400])
def test_rows_far_from_zero_and_rows_without_spread(cols, dtype):
    t, v = make(8, cols, dtype, True, 0, True, True, 3)
    t["r"] = stored(t["r"] * 0.0 + np.arange(8)[:, None], dtype)
    t["h"] = stored(np.where(np.arange(8)[:, None] % 2, t["h"] + 100.0, 3.0), dtype)
    check_fwd(8, cols, dtype, data=(t, v))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [40, 1000, 4096, 16400])
def test_what_is_not_a_number_stays_in_its_row(cols, dtype):
    torch = torch_mod()
    tt = torch_type(dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    r, h, dro, dy = (torch.randn(6, cols, generator=g, device="cuda").to(tt) for _ in range(4))
    r[1, cols // 2], h[3, 0], h[4, cols - 1] = float("nan"), float("inf"), float("nan")
    d = B.make_residual_norm_desc(6, cols, dtype, EPS)
    o, y, st = torch.empty_like(r), torch.empty_like(r), torch.empty(6, 4, device="cuda")
    B.residual_norm_fwd(d, r, h, None, None, None, None, None, None, o, y, st)
    bad = torch.isnan(y).any(1).cpu().tolist()
    assert bad == [False, True, False, True, True, False] and torch.isnan(y[3]).all() and torch.isnan(o[3]).all() and int(torch.isnan(o[1]).sum()) == 1
    dr, dh = torch.empty_like(r), torch.empty_like(r)
    B.residual_norm_bwd(d, o, h, None, None, None, None, None, st, dro, dy, dr, dh, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), workspace_bytes=1 << 20)
    assert torch.isnan(dr).any(1).cpu().tolist() == bad and torch.isfinite(dh[[0, 2, 5]]).all()


def test_without_rows():
    torch = torch_mod()
    d = B.make_residual_norm_desc(0, 100, wl.BF16)
    need = B.residual_norm_bwd_workspace_bytes(d)
    outs = [nan_vec(100) for _ in range(5)]
    B.residual_norm_bwd(d, None, None, None, None, None, None, None, None, None, None, None, None, None, *outs, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), need)
    assert all(bool((o == 0).all()) for o in outs)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,gate_rows", [(200, 7), (200, 1), (3000, 0), (16400, 50)])
def test_rows_far_apart(dtype, cols, gate_rows):
    """Offsets above 2^32 elements give what neighbouring rows give."""
    torch = torch_mod()
    tt, rows, ld = torch_type(dtype), 1100, 4_000_037
    g = torch.Generator(device="cuda").manual_seed(cols)
    near = {k: torch.randn(rows, cols, generator=g, device="cuda").to(tt) for k in ("r", "h", "dr_out", "dy")}
    gate = torch.randn(-(-rows // gate_rows), cols, generator=g, device="cuda").to(tt) if gate_rows else None
    vectors = [torch.randn(cols, generator=g, device="cuda") for _ in range(5)]
    # (three tensors far apart, each used twice)
    far = [torch.empty(rows * ld, dtype=tt, device="cuda").as_strided((rows, cols), (ld, 1)) for _ in range(3)]
    results = []
    for apart in (False, True):
        stride = ld if apart else None
        new = lambda: torch.empty(rows, cols, dtype=tt, device="cuda")  # noqa: E731
        r, h, y = far if apart else (new(), new(), new())
        r.copy_(near["r"]), h.copy_(near["h"])
        d = B.make_residual_norm_desc(rows, cols, dtype, EPS, False, True, gate_rows, True, stride, stride, cols if gate_rows else 0, stride)
        st = torch.empty(rows, 4, device="cuda")
        B.residual_norm_fwd(d, r, h, gate, *vectors, r, y, st)  # the sum over r
        results.append([r.clone(), y.clone(), st])
        need = B.residual_norm_bwd_workspace_bytes(d)
        dgate = torch.empty_like(gate) if gate_rows else None
        sums = [nan_vec(cols) for _ in range(5)]
        y.copy_(near["dy"])
        dh = torch.empty(rows * ld, dtype=tt, device="cuda").as_strided((rows, cols), (ld, 1)) if apart else new()
        B.residual_norm_bwd(d, r, h, gate, *vectors[:4], st, None, y, None, dh, dgate, *sums, torch.empty(need, dtype=torch.uint8, device="cuda"), need)
        results[-1] += [dh.clone(), *([dgate] if gate_rows else []), *sums]
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 40), (1000, 64), (700, 1000), (300, 9000), (40, 16400)])
def test_a_gate_for_more_rows_than_there_are(rows, cols, dtype):
    for gate_rows in (rows + 1, (1 << 31) - 1):
        kind = dict(gate_rows=gate_rows, sigmoid=True, post=cols % 3 != 0)
        check_fwd(rows, cols, dtype, **kind)
        # (the bound's roundings of a gate's sum: as many as it has rows)
        check_bwd(rows, cols, dtype, gate_rows=max(2, rows), sigmoid=True, post=kind["post"])
        torch = torch_mod()
        g = torch.Generator(device="cuda").manual_seed(rows)
        r, h, dro, dy = (torch.randn(rows, cols, generator=g, device="cuda").to(torch_type(dtype)) for _ in range(4))
        gate, st = torch.randn(1, cols, generator=g, device="cuda").to(r.dtype), torch.rand(rows, 4, generator=g, device="cuda")
        results = []
        for n in (max(2, rows), gate_rows):
            d = B.make_residual_norm_desc(rows, cols, dtype, EPS, gate_rows=n)
            need = B.residual_norm_bwd_workspace_bytes(d)
            dr, dh, dgate, sums = torch.empty_like(r), torch.empty_like(h), torch.empty_like(gate), [nan_vec(cols) for _ in range(5)]
            B.residual_norm_bwd(d, r, h, gate, None, None, None, None, st, dro, dy, dr, dh, dgate, *sums, torch.empty(need, dtype=torch.uint8, device="cuda"), need)
            results.append([dr, dh, dgate, *sums])
        assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 7, 255, 256, 257, 600])
@pytest.mark.parametrize("cols,kind", [(8200, dict(gate_rows=3)), (8193, dict(gate_rows=1, sigmoid=True)), (16384, dict(post=False, rms=True))])
def test_wide_rows_in_every_share_of_the_workgroups(cols, kind, rows, dtype):
    """Rows too wide for the column sums: as many workgroups as CUs take them in runs, whatever rows share a gate."""
    check_bwd(rows, cols, dtype, **kind)
