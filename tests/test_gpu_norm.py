"""Layer norm, its gradients and the row quantiser on the GPU against the 64-bit oracle.

Tolerances, from the arithmetic: a sum of n fp32 terms formed by threads and joined as a tree is off by at most
(terms of a thread + joins) units of 2^-24 of the sum of magnitudes; a thread adds at most cols / 64 terms (64 lanes at
least share a long row; short rows are at most 64 terms), a tree joins at most 16 times: STEPS below.  Everything else is a handful of roundings."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod
from rows_util import EPS32, ROUND, TINY, Rows, assert_close, nan_vec, stored, torch_type, vec

pytestmark = pytest.mark.gpu

DTYPES = [wl.F32, wl.F16, wl.BF16]
# rows, cols: one row and one column, around the vectors (4, 8), waves (64 lanes x vector) and workgroups, and longer than any register row
SHAPES = [(1, 1), (3, 2), (5, 7), (2, 8), (65, 15), (4, 16), (7, 31), (129, 33), (6, 64), (33, 100), (9, 127), (10, 192), (1, 255), (20, 384),
          (3, 511), (17, 513), (2, 1000), (5, 1024), (4, 2047), (3, 2056), (2, 4096), (3, 4099), (1, 8192), (2, 8200), (2, 16384), (1, 16391),
          (2, 40000), (1, 70001)]
EPS = 1e-5


def steps(cols):
    return 96 + cols / 64.0


def random_x(rows, cols, dtype, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, cols)) * rng.uniform(0.3, 3.0, size=(rows, 1)) + rng.normal(size=(rows, 1))
    return stored(x, dtype)


def norm_error(x, gamma, beta, eps):
    """Bounds of the errors of (value before rounding, mean, rstd), relative to nothing: per element and per row."""
    n = steps(x.shape[1])
    y, mean, rstd = ro.layernorm(x, gamma, beta, eps)
    e_mean = n * EPS32 * np.abs(x).mean(1)                       # of the sum, and the division
    var = ((x - mean[:, None]) ** 2).mean(1)
    dev = np.abs(x - mean[:, None]).mean(1)
    e_dev = e_mean + 2 * EPS32 * (np.abs(x).max(1) + np.abs(mean))   # of a difference x - mean
    e_var = 2 * dev * e_dev + e_dev ** 2 + n * EPS32 * var
    e_rstd = rstd * (0.5 * e_var / (var + eps) + 8 * EPS32) + rstd * 3 * (e_var / (var + eps)) ** 2
    g = np.abs(gamma) if gamma is not None else 1.0
    e_y = g * (rstd[:, None] * e_dev[:, None] + np.abs(x - mean[:, None]) * e_rstd[:, None]) + 8 * EPS32 * (np.abs(y) + (np.abs(beta) if beta is not None else 0.0))
    return y, mean, rstd, e_y * 1.01, e_mean * 1.01, e_rstd * 1.01


def check_fwd(rows, cols, dtype, ldx=None, ldy=None, start=0, affine=3, seed=0, x=None, eps=EPS, stats=True):
    rng = np.random.default_rng(seed + 1)
    x = random_x(rows, cols, dtype, seed) if x is None else x
    gamma = rng.normal(1, 0.3, cols).astype(np.float32).astype(np.float64) if affine & 1 else None
    beta = rng.normal(0, 0.3, cols).astype(np.float32).astype(np.float64) if affine & 2 else None
    X = Rows(rows, cols, torch_type(dtype), ldx, start, fill=float("nan")).set(x)
    Y = Rows(rows, cols, torch_type(dtype), ldy, start, fill=7.0)
    mean, rstd = nan_vec(rows), nan_vec(rows)
    d = B.make_norm_desc(rows, cols, dtype, eps, ldx, ldy)
    B.layernorm_fwd(d, X.ptr, None if gamma is None else vec(gamma), None if beta is None else vec(beta), Y.ptr,
                    mean if stats else None, rstd if stats else None)
    torch_mod().cuda.synchronize()
    y, m, r, ey, em, er = norm_error(x, gamma, beta, eps)
    assert_close(Y.host(), y, ey + ROUND[dtype] * np.abs(y) * 1.01 + TINY[dtype] + ROUND[dtype] * ey, "y")
    if stats:
        assert_close(mean.cpu().numpy(), m, em + 2 * EPS32 * np.abs(m), "mean")
        assert_close(rstd.cpu().numpy(), r, er + 2 * EPS32 * r, "rstd")
    assert Y.untouched()
    return X, Y


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_layernorm_fwd(rows, cols, dtype):
    check_fwd(rows, cols, dtype, affine=cols % 4 if rows > 2 else 3, seed=rows + cols)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,ldx,ldy,start", [(100, 103, 117, 1), (192, 193, 192, 3), (256, 512, 264, 5), (1000, 1001, 1003, 7), (4096, 4100, 4097, 2), (9, 20, 9, 1)])
def test_layernorm_fwd_of_slices_that_start_anywhere(cols, ldx, ldy, start, dtype):
    check_fwd(13, cols, dtype, ldx, ldy, start, seed=cols, stats=cols != 256)


@pytest.mark.parametrize("dtype", DTYPES)
def test_layernorm_fwd_many_short_rows(dtype):
    check_fwd(70001, 24, dtype, seed=5)


def test_layernorm_fwd_large_means_constant_rows_and_values_that_are_not_finite():
    rng = np.random.default_rng(4)
    x = stored(rng.normal(size=(6, 300)) + 500.0, wl.F32)  # the variance is taken around the mean
    x[1] = 3.0
    x[2] = 0.0
    check_fwd(6, 300, wl.F32, x=x)
    torch = torch_mod()
    x[3, 17], x[4, 2] = np.nan, np.inf
    X, Y = Rows(6, 300, torch.float32).set(x), Rows(6, 300, torch.float32)
    B.layernorm_fwd(B.make_norm_desc(6, 300), X.ptr, None, None, Y.ptr)
    y = Y.host()
    assert np.isnan(y[3]).all() and np.isnan(y[4]).all() and np.isfinite(y[[0, 1, 2, 5]]).all()
    # eps = 0 on a row without variance: 0 * inf
    B.layernorm_fwd(B.make_norm_desc(6, 300, eps=0.0), X.ptr, None, None, Y.ptr)
    assert np.isnan(Y.host()[2]).all()


def bwd_error(x, dy, gamma, mean, rstd):
    """The formula's result with bounds of what fp32 adds, from the statistics as they are handed over."""
    n = steps(x.shape[1])
    dx, dg, db = ro.layernorm_bwd(x, dy, gamma, mean, rstd)
    xh = (x - mean[:, None]) * rstd[:, None]
    e_xh = 3 * EPS32 * rstd[:, None] * (np.abs(x) + np.abs(mean[:, None]))
    g = np.abs(dy) * (np.abs(gamma) if gamma is not None else 1.0)
    c1, c2 = g.mean(1)[:, None], (g * np.abs(xh)).mean(1)[:, None]
    e_c1, e_c2 = (n + 4) * EPS32 * c1, (n + 4) * EPS32 * c2 + (g * e_xh).mean(1)[:, None]
    e_dx = rstd[:, None] * (e_c1 + np.abs(xh) * e_c2 + e_xh * c2 + 6 * EPS32 * (g + c1 + np.abs(xh) * c2))
    m = len(x) + 64  # rows are added one after the other at worst
    e_dg = (np.abs(dy) * e_xh).sum(0) + m * EPS32 * (np.abs(dy) * np.abs(xh)).sum(0)
    e_db = m * EPS32 * np.abs(dy).sum(0)
    return dx, dg, db, e_dx * 1.01, e_dg * 1.01, e_db * 1.01


def check_bwd(rows, cols, dtype, ldx=None, ldy=None, start=0, gamma=True, seed=0, want=7, in_place=False):
    rng = np.random.default_rng(seed + 9)
    x = random_x(rows, cols, dtype, seed)
    dy = stored(rng.normal(0, 0.5, size=(rows, cols)), dtype)
    g = rng.normal(1, 0.3, cols).astype(np.float32).astype(np.float64) if gamma else None
    _, mean, rstd = ro.layernorm(x, None, None, EPS) if rows else (None, np.zeros(0), np.zeros(0))
    mean, rstd = mean.astype(np.float32).astype(np.float64), rstd.astype(np.float32).astype(np.float64)
    X = Rows(rows, cols, torch_type(dtype), ldx, start, fill=float("nan")).set(x)
    DY = Rows(rows, cols, torch_type(dtype), ldy, start, fill=float("nan")).set(dy)
    DX = DY if in_place else Rows(rows, cols, torch_type(dtype), ldx, start, fill=7.0)
    d = B.make_norm_desc(rows, cols, dtype, EPS, ldx, ldy)
    need = B.layernorm_bwd_workspace_bytes(d)
    ws = torch_mod().full((max(need, 16),), 0xFF, dtype=torch_mod().uint8, device="cuda")
    dg, db = nan_vec(cols), nan_vec(cols)
    B.layernorm_bwd(d, X.ptr, DY.ptr, None if g is None else vec(g), vec(mean), vec(rstd), DX.ptr if want & 1 else None,
                    dg if want & 2 else None, db if want & 4 else None, ws, need)
    torch_mod().cuda.synchronize()
    if rows:
        dx, wg, wb, ex, eg, eb = bwd_error(x, dy, g, mean, rstd)
    else:
        wg = wb = np.zeros(cols)
        eg = eb = 0.0
    if want & 1 and rows:
        assert_close(DX.host(), dx, ex + ROUND[dtype] * (np.abs(dx) + ex) + TINY[dtype], "dx")
        assert DX.untouched()
    if want & 2:
        assert_close(dg.cpu().numpy(), wg, eg + 2 * EPS32 * np.abs(wg), "dgamma")
    if want & 4:
        assert_close(db.cpu().numpy(), wb, eb + 2 * EPS32 * np.abs(wb), "dbeta")
    return DX, dg, db


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_layernorm_bwd(rows, cols, dtype):
    check_bwd(rows, cols, dtype, gamma=cols % 3 != 0, seed=rows * 3 + cols)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(0, 17), (300, 64), (1111, 100), (700, 384), (2050, 33), (515, 1024), (260, 4096), (3000, 520)])
def test_layernorm_bwd_over_many_rows(rows, cols, dtype):
    check_bwd(rows, cols, dtype, seed=rows)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,ldx,ldy,start", [(100, 103, 117, 1), (192, 193, 192, 3), (256, 512, 264, 5), (1000, 1001, 1003, 7), (4096, 4100, 4097, 2), (9, 20, 9, 1)])
def test_layernorm_bwd_of_slices_that_start_anywhere(cols, ldx, ldy, start, dtype):
    check_bwd(21, cols, dtype, ldx, ldy, start, seed=cols)


@pytest.mark.parametrize("want", [1, 2, 4, 3, 5, 6])
@pytest.mark.parametrize("cols", [96, 3000, 70001])
def test_layernorm_bwd_of_some_gradients_only(want, cols):
    check_bwd(7, cols, wl.F16, seed=want, want=want)


@pytest.mark.parametrize("cols", [96, 3000, 70001])
def test_layernorm_bwd_over_dy(cols):
    check_bwd(37, cols, wl.BF16, seed=3, in_place=True)


def test_layernorm_bwd_agrees_with_differences_of_the_forward_pass():
    rows, cols, h = 5, 203, 1e-5
    rng = np.random.default_rng(8)
    x, v = random_x(rows, cols, wl.F32, 21), rng.normal(size=(rows, cols))
    dy = stored(rng.normal(size=(rows, cols)), wl.F32)
    gamma, beta = rng.normal(1, 0.3, cols).astype(np.float32).astype(np.float64), np.zeros(cols)
    X, DY, DX = (Rows(rows, cols, torch_type(wl.F32)) for _ in range(3))
    X.set(x), DY.set(dy)
    Y, mean, rstd, dg, db = Rows(rows, cols, torch_type(wl.F32)), nan_vec(rows), nan_vec(rows), nan_vec(cols), nan_vec(cols)
    d = B.make_norm_desc(rows, cols, wl.F32, EPS)
    B.layernorm_fwd(d, X.ptr, vec(gamma), vec(beta), Y.ptr, mean, rstd)
    ws = torch_mod().empty(max(16, B.layernorm_bwd_workspace_bytes(d)), dtype=torch_mod().uint8, device="cuda")
    B.layernorm_bwd(d, X.ptr, DY.ptr, vec(gamma), mean, rstd, DX.ptr, dg, db, ws, ws.numel())
    f = lambda x, g: (ro.layernorm(x, g, beta, EPS)[0] * dy).sum(1)  # noqa: E731
    want = (f(x + h * v, gamma) - f(x - h * v, gamma)) / (2 * h)
    # fp32 roundings of about a thousand terms of size 1, and h^2 of the differences
    assert np.allclose((DX.host() * v).sum(1), want, atol=1e-3, rtol=1e-4)
    gv = rng.normal(size=cols)
    want = (f(x, gamma + h * gv).sum() - f(x, gamma - h * gv).sum()) / (2 * h)
    assert abs(float((dg.cpu().numpy() * gv).sum()) - want) < 1e-2


# ---- rows to 8 bits --------------------------------------------------------------------------------------------------


def same_codes(q, scale, codes, scales, cols):
    got, padded = q.host(), B.row_stride(cols)
    assert np.array_equal(scale.cpu().numpy().view(np.uint32)[~np.isnan(scales)], scales.view(np.uint32)[~np.isnan(scales)])
    assert np.array_equal(np.isnan(scale.cpu().numpy()), np.isnan(scales))
    assert np.array_equal(got[:, :cols], codes)
    if q.ld >= padded:
        body = q.flat[q.start:q.start + q.rows * q.ld].view(q.rows, q.ld)
        assert bool((body[:, cols:padded] == 0).all())
    assert q.untouched(padded)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_rows_gives_the_definitions_codes(rows, cols, dtype):
    torch = torch_mod()
    x = random_x(rows, cols, dtype, rows + 2 * cols)
    ld = cols + (cols % 3)
    X = Rows(rows, cols, torch_type(dtype), ld, cols % 5, fill=float("inf")).set(x)
    Q = Rows(rows, cols, torch.int8, B.row_stride(cols) + 16 * (cols % 2), fill=99)
    scale = nan_vec(rows)
    B.quantize_rows(B.make_quant_desc(rows, cols, dtype, ld, Q.ld), X.ptr, Q.ptr, scale)
    same_codes(Q, scale, *ro.quantize_rows(x), cols)


@pytest.mark.parametrize("cols", [5, 300, 9000])
def test_quantize_rows_of_zeros_tiny_huge_and_values_that_are_not_finite(cols):
    torch = torch_mod()
    rng = np.random.default_rng(cols)
    x = rng.normal(size=(10, cols)).astype(np.float32).astype(np.float64)
    x[0] = 0.0
    x[1] *= 1e-38                  # magnitudes among the denormal numbers once divided by 127
    x[2] = stored(x[2] * 1e-44, wl.F32)
    x[3] = stored(x[3] * 1e38 / np.abs(x[3]).max() * 3.4, wl.F32)
    x[4, cols // 2] = np.nan
    x[5, cols - 1] = -np.inf
    x[6, 0] = np.inf
    x[7] = -0.0
    x[8] = np.arange(cols) % 255 - 127 + 0.5   # ties
    x[8, 0] = 127.0
    x[1] = stored(x[1], wl.F32)
    X = Rows(10, cols, torch.float32).set(x)
    Q = Rows(10, cols, torch.int8, B.row_stride(cols), fill=99)
    scale = nan_vec(10)
    B.quantize_rows(B.make_quant_desc(10, cols), X.ptr, Q.ptr, scale)
    codes, scales = ro.quantize_rows(x)
    same_codes(Q, scale, codes, scales, cols)
    assert np.isnan(scales[[4, 5, 6]]).all() and np.isfinite(scales[[0, 1, 2, 3, 7, 8, 9]]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 7), (40, 33), (20, 384), (3, 1001), (2, 4096), (2, 16391), (1, 70001)])
def test_layernorm_quant_is_the_two_calls(rows, cols, dtype):
    torch = torch_mod()
    rng = np.random.default_rng(cols)
    x = random_x(rows, cols, dtype, rows + cols)
    if rows > 4:
        x[3, 0] = np.nan
    X = Rows(rows, cols, torch_type(dtype), cols + 1, 1).set(x)
    gamma, beta = vec(rng.normal(1, 0.3, cols)), vec(rng.normal(0, 0.3, cols))
    Y = Rows(rows, cols, torch_type(dtype))
    Q = Rows(rows, cols, torch.int8, B.row_stride(cols), fill=99)
    scale = nan_vec(rows)
    B.layernorm_fwd(B.make_norm_desc(rows, cols, dtype, EPS, cols + 1, cols), X.ptr, gamma, beta, Y.ptr)
    B.layernorm_quant_fwd(B.make_norm_desc(rows, cols, dtype, EPS, cols + 1, Q.ld), X.ptr, gamma, beta, Q.ptr, scale)
    same_codes(Q, scale, *ro.quantize_rows(Y.host()), cols)


# many rows and few take different numbers of waves for a row; around the ends of waves and of pieces
WIDE = [(3, 1025), (600, 1025), (600, 1152), (514, 1537), (513, 2563), (5, 5120), (520, 5121), (515, 8193), (513, 9637), (2, 12289), (600, 1031), (2, 16383), (2, 17000), (1, 32768)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", WIDE)
def test_rows_of_any_number_of_waves(rows, cols, dtype):
    torch = torch_mod()
    check_fwd(rows, cols, dtype, cols + cols % 3, cols + 1, 1, seed=cols)
    x = random_x(rows, cols, dtype, rows + 2 * cols)
    x[rows // 2, cols - 1] = np.nan
    X = Rows(rows, cols, torch_type(dtype), cols + 1, 1, fill=float("inf")).set(x)
    Q = Rows(rows, cols, torch.int8, B.row_stride(cols) + 16, fill=99)
    scale = nan_vec(rows)
    B.quantize_rows(B.make_quant_desc(rows, cols, dtype, X.ld, Q.ld), X.ptr, Q.ptr, scale)
    same_codes(Q, scale, *ro.quantize_rows(x), cols)
    rng = np.random.default_rng(cols)
    gamma, beta = vec(rng.normal(1, 0.3, cols)), vec(rng.normal(0, 0.3, cols))
    Y = Rows(rows, cols, torch_type(dtype))
    B.layernorm_fwd(B.make_norm_desc(rows, cols, dtype, EPS, X.ld, cols), X.ptr, gamma, beta, Y.ptr)
    B.layernorm_quant_fwd(B.make_norm_desc(rows, cols, dtype, EPS, X.ld, Q.ld), X.ptr, gamma, beta, Q.ptr, scale)
    same_codes(Q, scale, *ro.quantize_rows(Y.host()), cols)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(600, 1025), (300, 2563), (70, 9637), (40, 16383)])
def test_layernorm_bwd_of_wide_rows(rows, cols, dtype):
    check_bwd(rows, cols, dtype, cols + 1, cols + 3, 1, seed=cols)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(600, 1152), (530, 1536), (270, 4097), (270, 5120), (260, 6143), (300, 8192), (257, 8193), (300, 12288), (258, 12289), (3, 16384), (2, 16385)])
def test_layernorm_bwd_of_rows_of_any_number_of_waves(rows, cols, dtype):
    check_bwd(rows, cols, dtype, seed=cols)
    check_bwd(min(rows, 5), cols, dtype, cols + 8, cols + 8, 0, seed=cols + 1, want=1, in_place=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 2, 40])
@pytest.mark.parametrize("cols", [1, 3, 4, 5, 7, 8, 9, 11])
def test_rows_of_less_than_a_piece_that_fill_their_tensor(rows, cols, dtype):
    """Nothing lies behind the last row, nor before the first."""
    check_fwd(rows, cols, dtype, seed=cols)
    check_bwd(rows, cols, dtype, seed=cols)


def test_offsets_beyond_32_bits():
    """Rows of tensors of 2.2e9 elements against the same rows on their own."""
    torch = torch_mod()
    rows, cols, ld = 20, 777, 110_000_000
    free, _ = torch.cuda.mem_get_info()
    assert free > 20 * 2 ** 30
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    own = torch.randn(rows, cols, generator=g, device="cuda").half()
    dy = torch.randn(rows, cols, generator=g, device="cuda").half()
    gamma, beta = torch.rand(cols, generator=g, device="cuda"), torch.rand(cols, generator=g, device="cuda")
    far, out = (torch.zeros(rows * ld, dtype=torch.float16, device="cuda").view(rows, ld) for _ in range(2))
    far[:, :cols] = own
    mean, rstd = nan_vec(rows), nan_vec(rows)
    near = torch.empty_like(own)
    B.layernorm_fwd(B.make_norm_desc(rows, cols, wl.F16, EPS), own, gamma, beta, near, mean, rstd)
    B.layernorm_fwd(B.make_norm_desc(rows, cols, wl.F16, EPS, ld, ld), far, gamma, beta, out)
    assert torch.equal(out[:, :cols], near)
    q = [torch.zeros(rows, B.row_stride(cols), dtype=torch.int8, device="cuda") for _ in range(2)]
    s = [nan_vec(rows) for _ in range(2)]
    B.quantize_rows(B.make_quant_desc(rows, cols, wl.F16), own, q[0], s[0])
    B.quantize_rows(B.make_quant_desc(rows, cols, wl.F16, ld), far, q[1], s[1])
    assert torch.equal(q[0], q[1]) and torch.equal(s[0], s[1])
    dx, res = torch.empty_like(own), []
    for x, d, o, l in ((own, dy, dx, cols), (far, dy, out, ld)):
        desc = B.make_norm_desc(rows, cols, wl.F16, EPS, l, cols)
        ws = torch.empty(max(16, B.layernorm_bwd_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
        dg, db = nan_vec(cols), nan_vec(cols)
        B.layernorm_bwd(desc, x, d, gamma, mean, rstd, o, dg, db, ws, ws.numel())
        res.append((o[:, :cols].clone(), dg, db))
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_gradients_of_a_row_of_more_columns_than_a_launch_joins():
    """2^27 columns: 16 threads for each of twice as many sums would be 2^32.  One row, so every sum is one product."""
    torch = torch_mod()
    cols = (1 << 27) + 70
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x, dy = (torch.randn(1, cols, generator=g, device="cuda").half() for _ in range(2))
    mean, rstd = torch.full((1,), 0.25, device="cuda"), torch.full((1,), 1.5, device="cuda")
    d = B.make_norm_desc(1, cols, wl.F16, EPS)
    ws = torch.empty(B.layernorm_bwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    dgamma, dbeta = nan_vec(cols), nan_vec(cols)
    B.layernorm_bwd(d, x, dy, None, mean, rstd, None, dgamma, dbeta, ws, ws.numel())
    assert torch.equal(dbeta, dy[0].float())
    # fp16 less a quarter has 24 bits at most, times 1.5 a rounding, times dy another
    want = dy[0].double() * ((x[0].double() - 0.25) * 1.5)
    assert bool(((dgamma.double() - want).abs() <= 4 * EPS32 * want.abs()).all())
