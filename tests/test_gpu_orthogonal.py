"""Newton-Schulz steps on the GPU against 64 bits.

The error of a step's rounded factors is carried through the following steps, so the bound is on the norm of the difference, relative to the result's.
With u half a step of the parts that are multiplied (fp16: 2^-11; two parts: 2^-22 for what is left out of a product and 2^-22 for the parts themselves), rounding a
factor moves it by u / sqrt(3) of its norm at most, at random.  A step rounds four factors (X twice, A, B), whose products are weighted by no more than 5 with the coefficients
used here (|b| + |c| s^2 for s up to 0.5, where s^2 is small, and |b s^2 + c s^4| < 3 up to 1.2): 2 * 5 u / sqrt(3) for the four together.  The steps that
follow move an error by the polynomial's slope, at most 2.1 in magnitude between 0.5 and 1.2 and below 1.6 in the mean over its range; errors of different steps are independent and
add as squares.  fp32 adds the roundings of its sums of n and m terms, 2^-24 sqrt(n + m) each, and those of X, which grow with the weak directions by a in a step,
a^steps 2^-24; the result is rounded once."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod
from rows_util import EPS32, ROUND, stored, torch_type

pytestmark = pytest.mark.gpu

DTYPES = [wl.F32, wl.F16, wl.BF16]
STEP = (3.4445, -4.7750, 2.0315)
CUBIC = (1.5, -0.5, 0.0)


def bound(dtype, rows, cols, steps, coefficients):
    u = 2.0 ** -11 if dtype == wl.BF16 else 2.0 ** -21
    grown = np.sqrt(sum(1.6 ** (2 * i) for i in range(steps)))
    return 2 * 5 * (u / np.sqrt(3) + EPS32 * np.sqrt(rows + cols)) * grown + abs(coefficients[0]) ** steps * EPS32 + ROUND[dtype]


def matrices(batch, rows, cols, dtype, kind, seed):
    rng = np.random.default_rng(seed + rows + 3 * cols)
    few = max(1, min(rows, cols) // 8)
    low = np.matmul(rng.normal(size=(batch, rows, few)), rng.normal(size=(batch, few, cols))) / np.sqrt(few)
    x = {"low": low, "full": rng.normal(size=(batch, rows, cols)), "mixed": low + 0.3 * rng.normal(size=(batch, rows, cols))}[kind]
    return stored(x * rng.uniform(1e-4, 1e-2, (batch, 1, 1)), dtype)


def check(batch, rows, cols, dtype, steps=5, kind="mixed", coefficients=STEP, pad=(0, 0), gap=(0, 0), start=0, inplace=False, seed=0):
    torch = torch_mod()
    x = matrices(batch, rows, cols, dtype, kind, seed)
    ldx, ldo = cols + pad[0], cols + (pad[0] if inplace else pad[1])
    sx, so = rows * ldx + gap[0], rows * ldo + (gap[0] if inplace else gap[1])
    tt = torch_type(dtype)

    def place(ld, stride, fill):
        flat = torch.full((start + batch * stride + 64,), fill, dtype=tt, device="cuda")
        return flat, flat[start:start + batch * stride].as_strided((batch, rows, cols), (stride, ld, 1), start)

    xf, xv = place(ldx, sx, float("nan"))
    xv.copy_(torch.from_numpy(x).to(tt))
    of, ov = (xf, xv) if inplace else place(ldo, so, 7.0)
    d = B.make_orthogonal_desc(rows, cols, dtype, batch, steps, coefficients, ldx=ldx, ldo=ldo, stride_x=sx, stride_o=so)
    need = B.orthogonalize_workspace_bytes(d)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    B.orthogonalize(d, xv.data_ptr(), ov.data_ptr(), ws, need)
    torch.cuda.synchronize()
    got = ov.double().cpu().numpy()
    for i in range(batch):
        want = ro.newton_schulz(x[i], steps, coefficients, 1e-7)
        off, norm = np.linalg.norm(got[i] - want), np.linalg.norm(want)
        assert off <= bound(dtype, rows, cols, steps, coefficients) * norm, (i, off / norm, bound(dtype, rows, cols, steps, coefficients))
    if not inplace:
        ov.fill_(7.0)
        assert bool((of == 7.0).all())


SIZES = [(1, 1, 1), (3, 1, 9), (2, 7, 1), (1, 16, 16), (5, 17, 33), (2, 64, 64), (3, 65, 200), (1, 128, 100), (2, 300, 129), (1, 257, 511), (1, 512, 512), (1, 700, 260), (24, 96, 384)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("batch,rows,cols", SIZES)
def test_matrices(batch, rows, cols, dtype):
    for kind in ("mixed", "full", "low"):
        if kind != "low" or min(rows, cols) >= 8:
            check(batch, rows, cols, dtype, kind=kind)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("steps,coefficients", [(1, STEP), (2, STEP), (6, STEP), (1, CUBIC), (8, CUBIC)])
def test_steps(steps, coefficients, dtype):
    check(2, 100, 72, dtype, steps, coefficients=coefficients)
    check(2, 60, 130, dtype, steps, coefficients=coefficients)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,gap,start", [((1, 3), (5, 0), 1), ((8, 0), (0, 9), 0), ((0, 7), (3, 3), 3)])
def test_strides(pad, gap, start, dtype):
    check(3, 50, 70, dtype, pad=pad, gap=gap, start=start)
    check(3, 70, 50, dtype, pad=pad, gap=gap, start=start)
    check(2, 50, 70, dtype, pad=pad, gap=gap, start=start, inplace=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(2048, 512), (1000, 3000), (2048, 2048)])
def test_large(rows, cols, dtype):
    check(1, rows, cols, dtype)


def test_many_small_matrices():
    check(1000, 8, 12, wl.F32)


@pytest.mark.parametrize("dtype", DTYPES)
def test_sizes_of_values(dtype):
    """From the smallest normal numbers to the largest: the result does not depend on the update's size, but for eps."""
    torch = torch_mod()
    x = torch.randn(3, 40, 60, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    small, large = (1e-4, 1e4) if dtype == wl.F16 else (1e-36, 1e36)
    x = (x * torch.tensor([small, 1.0, large], device="cuda").view(3, 1, 1)).to(torch_type(dtype))
    y = torch.empty_like(x)
    d = B.make_orthogonal_desc(40, 60, dtype, 3, eps=0.0)
    n = B.orthogonalize_workspace_bytes(d)
    B.orthogonalize(d, x, y, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    for i in range(3):
        want = ro.newton_schulz(x[i].double().cpu().numpy(), 5, STEP, 0.0)
        assert np.linalg.norm(y[i].double().cpu().numpy() - want) <= bound(dtype, 40, 60, 5, STEP) * np.linalg.norm(want)


def test_zeros_and_what_is_not_a_number():
    torch = torch_mod()
    x = torch.randn(4, 30, 50, device="cuda")
    x[0], x[1, 3, 4], x[2, 0, 0] = 0.0, float("nan"), float("inf")
    y = torch.empty_like(x)
    d = B.make_orthogonal_desc(30, 50, wl.F32, 4)
    n = B.orthogonalize_workspace_bytes(d)
    B.orthogonalize(d, x, y, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    assert bool((y[0] == 0).all()) and bool(torch.isnan(y[1]).all()) and bool(torch.isnan(y[2]).all()) and bool(torch.isfinite(y[3]).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_matrix_for_all_of_a_batch(dtype):
    torch = torch_mod()
    x = torch.randn(40, 24, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(torch_type(dtype))
    y = torch.empty(5, 40, 24, dtype=x.dtype, device="cuda")
    d = B.make_orthogonal_desc(40, 24, dtype, 5, stride_x=0)
    n = B.orthogonalize_workspace_bytes(d)
    B.orthogonalize(d, x, y, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    want = ro.newton_schulz(x.double().cpu().numpy(), 5, STEP, 1e-7)
    assert all(torch.equal(y[0], y[i]) for i in range(5))
    assert np.linalg.norm(y[0].double().cpu().numpy() - want) <= bound(dtype, 40, 24, 5, STEP) * np.linalg.norm(want)


def test_more_matrices_than_a_launch_takes():
    torch = torch_mod()
    batch = 33000
    x = torch.randn(batch, 5, 9, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda")
    y = torch.empty_like(x)
    d = B.make_orthogonal_desc(5, 9, wl.F32, batch)
    n = B.orthogonalize_workspace_bytes(d)
    B.orthogonalize(d, x, y, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    for i in (0, 1, 32767, 32768, 32999):
        want = ro.newton_schulz(x[i].double().cpu().numpy(), 5, STEP, 1e-7)
        assert np.linalg.norm(y[i].double().cpu().numpy() - want) <= bound(wl.F32, 5, 9, 5, STEP) * np.linalg.norm(want)
    assert bool(torch.isfinite(y).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_far_apart(dtype):
    """Offsets above 2^32 elements."""
    torch = torch_mod()
    ld, rows, cols = (1 << 23) + 3, 600, 40
    tt = torch_type(dtype)
    x, y = (torch.empty(rows * ld, dtype=tt, device="cuda").as_strided((rows, cols), (ld, 1)) for _ in range(2))
    x.copy_(torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda").to(tt))
    d = B.make_orthogonal_desc(rows, cols, dtype, ldx=ld, ldo=ld)
    n = B.orthogonalize_workspace_bytes(d)
    B.orthogonalize(d, x, y, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    want = ro.newton_schulz(x.double().cpu().numpy(), 5, STEP, 1e-7)
    assert np.linalg.norm(y.double().cpu().numpy() - want) <= bound(dtype, rows, cols, 5, STEP) * np.linalg.norm(want)


@pytest.mark.parametrize("rows,cols,steps", [(45, 118, 6), (23, 18, 6), (166, 30, 6), (64, 64, 5), (24, 300, 4), (300, 260, 5), (512, 512, 6), (600, 600, 5)])
def test_bf16_results_are_off_by_little_more_than_their_rounding(rows, cols, steps):
    """The rounding alone is 2^-8 / sqrt(3) of a step at most, 1.7e-3 at random mantissas: 1.35 times that here."""
    torch = torch_mod()
    x = matrices(2, rows, cols, wl.BF16, "mixed", 3)
    t = torch.from_numpy(x).to(torch.bfloat16).cuda()
    y = torch.empty_like(t)
    d = B.make_orthogonal_desc(rows, cols, wl.BF16, 2, steps)
    n = B.orthogonalize_workspace_bytes(d)
    B.orthogonalize(d, t, y, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    for i in range(2):
        want = ro.newton_schulz(x[i], steps, STEP, 1e-7)
        rounded = torch.from_numpy(want).to(torch.bfloat16).double().numpy()
        off = np.linalg.norm(y[i].double().cpu().numpy() - want)
        assert off <= 1.35 * np.linalg.norm(rounded - want), (off / np.linalg.norm(rounded - want))
