"""Linear layers on the GPU, forward and backward, against 64 bits.

Bounds: a sum of K products in fp32 is off by at most K + 2 roundings of the magnitudes it adds up (the parts of fp32 operands that are
left out are below 2^-25 of each product and their splitting below 2^-27: one more); activations move an error by their slope, at most 1.13, and add
a few roundings of their own (exp of z is off by |z| roundings); then one rounding to the type."""
import itertools

import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod
from rows_util import EPS32, ROUND, TINY, Rows, assert_close, nan_vec, stored, torch_type, vec

pytestmark = pytest.mark.gpu

DTYPES = [wl.F32, wl.F16, wl.BF16]
ACTS = ["none", "relu", "gelu", "silu"]


def workspace(need):
    torch = torch_mod()
    # whatever a workspace holds must not matter: NaN in every type
    return torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")


def act_tol(z, tol_z):
    return 1.13 * tol_z + EPS32 * (8 + 2 * np.abs(z)) * np.abs(z)


def slope_tol(z):
    return EPS32 * (16 + 4 * np.abs(z))


def check_fwd(rows, N, K, dtype, act="none", bias=True, residual=False, pre=False, pad=(0, 0, 0, 0), start=0, seed=0, inplace=False, stream=None, sigma=1.0):
    torch = torch_mod()
    rng = np.random.default_rng(seed + rows + 7 * N + 13 * K)
    tt, fill = torch_type(dtype), float("nan")
    x, w = stored(sigma * rng.normal(size=(rows, K)), dtype), stored(rng.normal(size=(N, K)) * K ** -0.5, dtype)
    b = rng.normal(size=N).astype(np.float32) if bias else None
    r = stored(rng.normal(size=(rows, N)), dtype) if residual else None
    X, W = Rows(rows, K, tt, K + pad[0], start, fill).set(x), Rows(N, K, tt, K + pad[1], start, fill).set(w)
    Y = Rows(rows, N, tt, N + pad[3], start, 7.0)
    Z = Rows(rows, N, tt, N + pad[3], start, 5.0) if pre else None
    R = Y if inplace else Rows(rows, N, tt, N + pad[2], start, fill) if residual else None
    if residual:
        R.set(r)
    d = B.make_linear_desc(rows, N, K, dtype, act, X.ld, W.ld, R.ld if residual else None, Y.ld)
    need = B.linear_workspace_bytes(d)
    B.linear_fwd(d, X.ptr, W.ptr, None if b is None else vec(b), R.ptr if residual else None, Y.ptr, Z.ptr if pre else None, workspace(need), need, stream)
    torch.cuda.synchronize()
    v, z, size = ro.linear(x, w, None if b is None else b.astype(np.float64), r, act)
    tol_z = (K + 3) * EPS32 * size
    if pre:
        assert_close(Z.host(), z, tol_z + ROUND[dtype] * (np.abs(z) + tol_z) + TINY[dtype], "pre")
        assert Z.untouched()
    tol = act_tol(z, tol_z) if act != "none" else tol_z
    if residual:
        tol = tol + EPS32 * (np.abs(v) + tol)
    assert_close(Y.host(), v, tol + ROUND[dtype] * (np.abs(v) + tol) + TINY[dtype], "out")
    assert Y.untouched()
    return B.linear_form(d, X.ptr, W.ptr)


def check_bwd(rows, N, K, dtype, act="none", pad=(0, 0, 0), start=0, seed=0, want=("dx", "dw", "dbias"), sigma=1.0):
    torch = torch_mod()
    rng = np.random.default_rng(seed + rows + 7 * N + 13 * K)
    tt, fill = torch_type(dtype), float("nan")
    x, w = stored(rng.normal(size=(rows, K)), dtype), stored(rng.normal(size=(N, K)) * K ** -0.5, dtype)
    z, g = stored(1.5 * rng.normal(size=(rows, N)), dtype), stored(sigma * rng.normal(size=(rows, N)), dtype)
    X, W = Rows(rows, K, tt, K + pad[0], start, fill).set(x), Rows(N, K, tt, K + pad[1], start, fill).set(w)
    Z, G = Rows(rows, N, tt, N + pad[2], start, fill).set(z), Rows(rows, N, tt, N + pad[2], start, fill).set(g)
    DX, DW, DB = Rows(rows, K, tt, K + pad[0], start, 7.0), Rows(N, K, tt, K + pad[1], start, 7.0), nan_vec(N)
    d = B.make_linear_desc(rows, N, K, dtype, act, X.ld, W.ld, None, G.ld)
    need = B.linear_bwd_workspace_bytes(d)
    out = [DX.ptr if "dx" in want else None, DW.ptr if "dw" in want else None, DB if "dbias" in want else None]
    B.linear_bwd(d, X.ptr if "dw" in want else None, W.ptr if "dx" in want else None, None if act == "none" else Z.ptr, G.ptr, *out, workspace(need), need)
    torch.cuda.synchronize()
    dx, dw, db = ro.linear_bwd(x, w, z, g, act)
    # the gradient at the sum, and how far off it is before and after its rounding to the type (fp32: to three bf16 parts)
    slope = ro.activation(z, act)[1]
    dz = g * slope
    off = np.abs(g) * slope_tol(z) + EPS32 * np.abs(dz) if act != "none" else 0.0 * np.abs(dz)
    rounded = off + (ROUND[dtype] * (np.abs(dz) + off) + TINY[dtype] if act != "none" and dtype != wl.F32 else 0.0)
    mag = np.abs(dz) + rounded
    for name, got, ref, n, size, moved in (("dx", DX, dx, N, mag @ np.abs(w), rounded @ np.abs(w)), ("dw", DW, dw, rows, mag.T @ np.abs(x), rounded.T @ np.abs(x))):
        if name in want:
            tol = (n + 3) * EPS32 * size + moved
            assert_close(got.host(), ref, tol + ROUND[dtype] * (np.abs(ref) + tol) + TINY[dtype], name)
        assert got.untouched(written=None if name in want else 0)
    if "dbias" in want:
        assert_close(DB.cpu().numpy(), db, (rows + 3) * EPS32 * mag.sum(0) + off.sum(0), "dbias")
    return [B.linear_form(d, X.ptr, W.ptr, i) for i in (1, 2)]


SMALL = [(1, 1, 1), (1, 10, 17), (2, 16, 64), (3, 33, 63), (5, 100, 128), (16, 130, 65), (17, 257, 300), (31, 64, 1001), (33, 48, 40), (65, 15, 129), (100, 200, 72), (129, 129, 65)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K", SMALL)
def test_small_forward(rows, N, K, dtype):
    for i, act in enumerate(ACTS):
        check_fwd(rows, N, K, dtype, act, bias=i != 1, residual=i % 2 == 1, pre=i >= 2, seed=i)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K", SMALL)
def test_small_backward(rows, N, K, dtype):
    for i, act in enumerate(ACTS):
        check_bwd(rows, N, K, dtype, act, seed=i)


LARGE = [(1, 4096, 4096), (5, 1000, 9216), (20, 1000, 4096), (16, 16, 16384), (64, 2048, 1024), (200, 1003, 999), (777, 1283, 1001), (256, 256, 128), (257, 255, 129),
         (512, 512, 512), (1000, 128, 4096), (1300, 1111, 640), (2048, 768, 1600), (3380, 1536, 384)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K", LARGE)
def test_forward(rows, N, K, dtype):
    i = rows + N + K + dtype
    check_fwd(rows, N, K, dtype, ACTS[i % 4], bias=i % 3 != 0, residual=i % 2 == 0, pre=i % 5 < 2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K", LARGE + [(9000, 64, 96), (2000, 3001, 200), (300, 9001, 64)])
def test_backward(rows, N, K, dtype):
    check_bwd(rows, N, K, dtype, ACTS[(rows + N + K + dtype) % 4])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,start", list(itertools.product([(8, 16, 8, 8), (1, 0, 3, 5), (0, 3, 0, 1), (7, 7, 1, 0)], [0, 1, 8])))
def test_strides_and_starts(dtype, pad, start):
    for rows, N, K in ((3, 37, 72), (70, 136, 200), (300, 264, 136)):
        check_fwd(rows, N, K, dtype, "relu", residual=True, pre=True, pad=pad, start=start)
        check_bwd(rows, N, K, dtype, "relu", pad=(pad[0], pad[1], pad[3]), start=start)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("want", [("dx",), ("dw",), ("dbias",), ("dx", "dbias"), ("dw", "dbias"), ("dx", "dw")])
def test_gradients_that_are_asked_for(dtype, want):
    for act, pad in (("none", 0), ("none", 3), ("gelu", 0)):
        check_bwd(150, 72, 136, dtype, act, pad=(0, 0, pad), want=want)


# (which product, rows, N, K, elements the first operand starts at) -> the form that has to be taken
FORMS = {
    "rows16": (0, 9, 40, 200, 0), "rows16_any": (0, 9, 41, 201, 1), "rows32": (0, 21, 40, 136, 0), "rows32_any": (0, 21, 41, 135, 1), "rows64": (0, 45, 72, 200, 0),
    "rows64_any": (0, 45, 73, 201, 1), "rows32_split16": (0, 20, 8, 9000, 0), "rows32_any_split16": (0, 20, 8, 9000, 1), "rows64_split16": (0, 40, 8, 9000, 0),
    "rows64_any_split12": (0, 130, 100, 9000, 1),
}
FORMS16 = {
    "tile64x64": (0, 700, 1032, 40, 0), "tile128x128": (0, 1000, 1032, 72, 0), "tile192x192": (0, 2000, 2056, 136, 0), "tile256x256": (0, 3000, 3080, 72, 0),
    "tile64x64_any": (0, 1100, 776, 40, 1), "tile128x128_any": (0, 2000, 1032, 72, 1), "tile256x256+tile128x128": (0, 5200, 3080, 40, 0),
    "tile256x256+tile192x192": (0, 5200, 4104, 24, 0), "tile64x64_any_split13": (0, 40, 8, 4104, 1), "tile128x128_split16": (0, 700, 136, 9000, 0),
    "tile128x128_any_split13": (0, 200, 1032, 4104, 1),
    "1 tile64x64": (1, 30, 40, 24, 0), "1 tile128x128": (1, 1000, 40, 1032, 0), "1 tile192x192": (1, 2000, 72, 2056, 0), "1 tile256x256": (1, 2600, 40, 4104, 0),
    "1 tile256x256+tile128x128": (1, 4100, 40, 4104, 0), "1 tile128x128_any": (1, 2000, 40, 1032, 1), "1 tile64x64_any_split13": (1, 3, 4104, 16, 1),
    "1 tile128x128_split13": (1, 1, 4104, 2056, 0), "2 tile64x64": (2, 40, 24, 72, 0), "2 tile128x128": (2, 40, 1000, 1032, 0), "2 tile192x192": (2, 72, 2056, 2056, 0),
    "2 tile256x256": (2, 40, 3080, 4104, 0), "2 tile256x256+tile128x128": (2, 40, 4104, 4104, 0), "2 tile128x128_any": (2, 40, 1000, 2056, 1),
    "2 tile64x64_any_split13": (2, 4100, 8, 16, 1), "2 tile128x128_split13": (2, 4100, 8, 2056, 0),
}
FORMS32 = {
    "split_tile64x64": (0, 700, 1000, 40, 1), "split_tile128x128": (0, 2000, 1032, 72, 1), "split_tile256x128": (0, 3000, 2056, 136, 0),
    "split_tile256x128+split_tile128x128": (0, 2600, 4104, 40, 0), "split_tile256x128+split_tile64x64": (0, 4100, 2056, 24, 1),
    "1 split_tile64x64": (1, 30, 40, 24, 1), "1 split_tile128x128": (1, 2000, 40, 1032, 0), "1 split_tile256x128": (1, 2000, 72, 2056, 0),
    "1 split_tile256x128+split_tile128x128": (1, 2600, 40, 4104, 1), "2 split_tile64x64": (2, 40, 24, 72, 0), "2 split_tile128x128": (2, 40, 1000, 2056, 1),
    "2 split_tile256x128": (2, 40, 2056, 2056, 0), "2 split_tile256x128+split_tile64x64": (2, 40, 4104, 2056, 0),
}


@pytest.mark.parametrize("dtype,name", [(t, n) for t in DTYPES for n in {**FORMS, **(FORMS32 if t == wl.F32 else FORMS16)} if (t, n) != (wl.F32, "rows64_any_split12")])
def test_every_form(dtype, name):
    which, rows, N, K, start = {**FORMS, **FORMS16, **FORMS32}[name]
    pad = -K % 8
    if which == 0:
        assert check_fwd(rows, N, K, dtype, "relu", residual=True, pre=True, inplace=True, pad=(pad, pad, -N % 8, -N % 8), start=start) == name
    else:
        got = check_bwd(rows, N, K, dtype, "relu", pad=(pad, pad, -N % 8), start=start, want=("dx",) if which == 1 else ("dw",))
        assert got[which - 1] == name.split()[1]


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_at_activations_give_the_limits(dtype):
    """A large sum rounds to an infinity in fp16: the slope there is the limit."""
    torch = torch_mod()
    inf, nan = float("inf"), float("nan")
    z = np.array([inf, -inf, nan, 0.0, -0.0, 1e4, -1e4, 100.0, -100.0, 17.0, -17.0, 15.0, -15.0, 3.0, -3.0, 6e4], dtype=np.float32)
    n = len(z)
    limits = {"relu": ([inf, 0.0], [1.0, 0.0]), "gelu": ([inf, 0.0], [1.0, 0.0]), "silu": ([inf, 0.0], [1.0, 0.0])}
    tt = torch_type(dtype)
    for act, (values, slopes) in limits.items():
        x, w = torch.ones(1, 1, dtype=tt, device="cuda"), torch.zeros(n, 1, dtype=tt, device="cuda")
        d = B.make_linear_desc(1, n, 1, dtype, act)
        out, pre = torch.empty(1, n, dtype=tt, device="cuda"), torch.empty(1, n, dtype=tt, device="cuda")
        B.linear_fwd(d, x, w, vec(z), None, out, pre)
        zs = stored(z, dtype)
        assert np.array_equal(pre.double().cpu().numpy()[0], zs, equal_nan=True)
        with np.errstate(invalid="ignore"):
            want, _ = ro.activation(z.astype(np.float64), act)
            _, slope = ro.activation(zs, act)
        want[:2], slope[:2] = values, slopes
        fin = np.where(np.isfinite(z), z, 0.0).astype(np.float64)
        tol = act_tol(fin, 0.0)
        assert_close(out.double().cpu().numpy()[0], want, tol + ROUND[dtype] * (np.abs(np.where(np.isfinite(want), want, 0.0)) + tol) + TINY[dtype], act)
        db = nan_vec(n)
        need = B.linear_bwd_workspace_bytes(d)
        B.linear_bwd(d, None, None, pre, torch.ones_like(out), None, None, db, workspace(need), need)
        assert_close(db.cpu().numpy(), slope, slope_tol(np.where(np.isfinite(zs), np.minimum(np.abs(zs), 20.0), 0.0)) + EPS32, "slope of " + act)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K,start", [(9, 40, 72, 0), (9, 41, 73, 1), (60, 300, 264, 0), (700, 1032, 136, 0), (700, 1031, 136, 1), (2000, 2056, 72, 0)])
def test_what_is_not_a_number_stays_in_its_row_and_column(dtype, rows, N, K, start):
    torch = torch_mod()
    tt, nan = torch_type(dtype), float("nan")
    rng = np.random.default_rng(5)
    X, W = Rows(rows, K, tt, K, start, nan).set(rng.normal(size=(rows, K))), Rows(N, K, tt, K, start, nan).set(rng.normal(size=(N, K)))
    G = Rows(rows, N, tt, N, start, nan).set(rng.normal(size=(rows, N)))
    at, col, k = rows // 2, N // 3, K - 1
    X.view[at, k], W.view[col, 0] = nan, float("inf")
    Y, DX, DW, DB = Rows(rows, N, tt, N, start, 7.0), Rows(rows, K, tt, K, start, 7.0), Rows(N, K, tt, K, start, 7.0), nan_vec(N)
    d = B.make_linear_desc(rows, N, K, dtype)
    need = B.linear_workspace_bytes(d)
    B.linear_fwd(d, X.ptr, W.ptr, None, None, Y.ptr, None, workspace(need), need)
    bad = ~np.isfinite(Y.host())
    assert bad[at].all() and bad[:, col].all() and bad.sum() == rows + N - 1
    G.view[at, 1] = nan
    need = B.linear_bwd_workspace_bytes(d)
    B.linear_bwd(d, X.ptr, W.ptr, None, G.ptr, DX.ptr, DW.ptr, DB, workspace(need), need)
    bad = ~np.isfinite(DX.host())
    assert bad[at].all() and bad[:, 0].all() and bad.sum() == rows + K - 1  # the row of the NaN, the column of the infinity
    bad = ~np.isfinite(DW.host())
    assert bad[1].all() and bad[:, k].all() and bad.sum() == N + K - 1
    assert np.flatnonzero(~np.isfinite(DB.cpu().numpy())).tolist() == [1]


def spread(rows, cols, tt, ld, values):
    """A tensor whose rows lie `ld` apart, of `values`; nothing else of its memory is written."""
    torch = torch_mod()
    t = torch.empty(rows * ld, dtype=tt, device="cuda").as_strided((rows, cols), (ld, 1))
    return t.copy_(torch.from_numpy(values).to(tt))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K,ld", [(1100, 40, 24, (1 << 22) + 8), (1100, 264, 136, (1 << 22) + 3), (40, 1100, 72, (1 << 22) - 8), (1100, 1100, 40, (1 << 22) - 8)])
def test_rows_far_apart(dtype, rows, N, K, ld):
    """Offsets above 2^32 elements, in every tensor."""
    torch = torch_mod()
    tt = torch_type(dtype)
    rng = np.random.default_rng(rows + N)
    x, w, g = (stored(rng.normal(size=s), dtype) for s in ((rows, K), (N, K), (rows, N)))
    X, W, R = spread(rows, K, tt, ld, x), spread(N, K, tt, ld, w), spread(rows, N, tt, ld, g)
    out = spread(rows, N, tt, ld, np.zeros((rows, N)))
    d = B.make_linear_desc(rows, N, K, dtype, "none", ld, ld, ld, ld)
    need = B.linear_workspace_bytes(d)
    B.linear_fwd(d, X, W, None, R, out, None, workspace(need), need)
    v, z, size = ro.linear(x, w, None, g, "none")
    tol = (K + 4) * EPS32 * (size + np.abs(g))
    assert_close(out.double().cpu().numpy(), v, tol + ROUND[dtype] * (np.abs(v) + tol) + TINY[dtype], "out")
    need = B.linear_bwd_workspace_bytes(d)
    dw = spread(N, K, tt, ld, np.zeros((N, K)))
    B.linear_bwd(d, X, W, None, R, out.as_strided((rows, K), (ld, 1)), dw, None, workspace(need), need)  # (dx where out was)
    for got, ref, n, size in ((out.as_strided((rows, K), (ld, 1)), g @ w, N, np.abs(g) @ np.abs(w)), (dw, g.T @ x, rows, np.abs(g).T @ np.abs(x))):
        tol = (n + 3) * EPS32 * size
        assert_close(got.double().cpu().numpy(), ref, tol + ROUND[dtype] * (np.abs(ref) + tol) + TINY[dtype], "gradient")


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_without_rows(dtype):
    torch = torch_mod()
    d = B.make_linear_desc(0, 30, 70, dtype, "gelu", ldw=73)
    DW, DB = Rows(30, 70, torch_type(dtype), 73, 1, 7.0), nan_vec(30)
    B.linear_bwd(d, None, None, None, None, None, DW.ptr, DB)
    assert not DW.host().any() and DW.untouched() and bool((DB == 0).all())


def test_calls_give_the_same_bits():
    """Sums are added in one order, shared reductions too."""
    torch = torch_mod()
    for rows, N, K, dtype in ((20, 1000, 4096, wl.F32), (700, 136, 9000, wl.BF16), (3000, 100, 200, wl.F16)):
        tt = torch_type(dtype)
        x, w, g = (torch.randn(s, device="cuda").to(tt) for s in ((rows, K), (N, K), (rows, N)))
        d = B.make_linear_desc(rows, N, K, dtype, "gelu")
        a, b = B.linear_workspace_bytes(d), B.linear_bwd_workspace_bytes(d)
        results = []
        for _ in range(3):
            out, pre, dx, dw, db = torch.empty_like(g), torch.empty_like(g), torch.empty_like(x), torch.empty_like(w), nan_vec(N)
            B.linear_fwd(d, x, w, None, None, out, pre, workspace(a), a)
            B.linear_bwd(d, x, w, pre, g, dx, dw, db, workspace(b), b)
            results.append((out, pre, dx, dw, db))
        for again in results[1:]:
            assert all(torch.equal(p, q) for p, q in zip(results[0], again))


@pytest.mark.parametrize("start", [0, 1])
@pytest.mark.parametrize("rows,N,K", [(1000, 300, 2000), (1300, 1111, 640), (600, 1000, 1000), (2, 4100, 3001)])
def test_fp32_gradients_of_shared_reductions(rows, N, K, start):
    forms = check_bwd(rows, N, K, wl.F32, "silu", start=start)
    assert any("_split" in f[5:] for f in forms)


def test_fp32_operands_that_parts_do_not_hold():
    """As documented: of small operands what lies below 2^-126 counts as zero, and infinities give NaN in tiles, themselves in few rows."""
    torch = torch_mod()
    rng = np.random.default_rng(2)
    inf = float("inf")
    for rows, N, K in ((3000, 2056, 136), (4, 40, 64)):
        x, w = stored(2.0 ** -112 * rng.normal(size=(rows, K)), wl.F32), stored(rng.normal(size=(N, K)), wl.F32)
        X, W = Rows(rows, K, torch.float32, fill=inf).set(x), Rows(N, K, torch.float32, fill=inf).set(w)
        Y = Rows(rows, N, torch.float32, fill=7.0)
        d = B.make_linear_desc(rows, N, K, wl.F32)
        need = B.linear_workspace_bytes(d)
        B.linear_fwd(d, X.ptr, W.ptr, None, None, Y.ptr, None, workspace(need), need)
        _, z, size = ro.linear(x, w, None, None, "none")
        # (each of x's three parts may lose as much as one that rounds to the smallest normal number)
        assert_close(Y.host(), z, (K + 4) * EPS32 * size + 2 * 2.0 ** -126 * np.abs(w).sum(1), "small")
        tiles = B.linear_form(d, X.ptr, W.ptr).startswith("split_")
        assert tiles == (rows == 3000)
        X.set(np.ones((rows, K))), W.set(np.ones((N, K)))
        X.view[1, 3] = inf
        B.linear_fwd(d, X.ptr, W.ptr, None, None, Y.ptr, None, workspace(need), need)
        got = Y.host()
        assert (np.isnan(got[1]) if tiles else np.isposinf(got[1])).all() and (np.delete(got, 1, 0) == K).all()


# rows, N, K, elements the operands start at -> the form that has to be taken
WIDE = {"rows32x64": (21, 12305, 296, 0), "rows64x64": (45, 12345, 1032, 0), "rows16x32_any": (9, 6157, 301, 1), "rows32x32_any": (29, 6170, 273, 1)}


@pytest.mark.parametrize("name", WIDE)
def test_few_fp32_rows_over_many_outputs(name):
    rows, N, K, start = WIDE[name]
    for act, r in (("none", rows), ("silu", rows - 4)):
        assert check_fwd(r, N, K, wl.F32, act, residual=True, pre=act == "silu", inplace=act == "none", pad=(0, 0, 3, 3), start=start, seed=r) == name
    # ... and rows that lie apart
    pad = 8 if start == 0 else 5
    assert check_fwd(rows, N, K, wl.F32, "relu", pad=(pad, 2 * pad, 0, 1), start=start) == name


@pytest.mark.parametrize("rows,N,K,start", [(1, 300, 16384, 0), (9, 6157, 4099, 1), (24, 12305, 4096, 0), (20, 400, 9001, 1), (48, 300, 4096, 0)])
def test_long_fp32_sums_of_few_rows(rows, N, K, start):
    """A sum is formed in eight chains of K / 8 terms or more of them.  At random signs the sums within a chain of n terms of size s grow as s sqrt(k), a rounding of which
    is 2^-24 / sqrt(3) of it: 2^-24 s n / sqrt(6) in all, and for all chains 2^-24 sqrt(K / 8) / sqrt(6) of the result's norm."""
    torch = torch_mod()
    rng = np.random.default_rng(rows + K)
    x, w = stored(rng.normal(size=(rows, K)), wl.F32), stored(rng.normal(size=(N, K)) * K ** -0.5, wl.F32)
    X, W, Y = Rows(rows, K, torch.float32, start=start).set(x), Rows(N, K, torch.float32, start=start).set(w), torch.empty(rows, N, device="cuda")
    d = B.make_linear_desc(rows, N, K, wl.F32)
    need = B.linear_workspace_bytes(d)
    B.linear_fwd(d, X.ptr, W.ptr, None, None, Y, None, workspace(need), need)
    assert B.linear_form(d, X.ptr, W.ptr).startswith("rows")
    want = x @ w.T
    assert np.linalg.norm(Y.double().cpu().numpy() - want) <= EPS32 * (np.sqrt(K / 8) / np.sqrt(6) + 1) * np.linalg.norm(want)
