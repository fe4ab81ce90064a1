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
