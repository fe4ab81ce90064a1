"""Newton-Schulz steps on bf16 matrices of many spectra: results are off by their own rounding and hardly more.

A result w + e that is rounded once is off by no more than the rounding of w and two times e (where e moves a value over a border it moves the rounded one by more than itself, but not in
the mean).  e by the arithmetic of test_gpu_orthogonal.py's bound for products of two parts (u = 2^-21) and fp32 sums: for five steps of sides of some 600 together 1.5e-4 of the result's
norm, a tenth of a rounding of 1.66e-3; its signs are random, so as squares it adds half a percent.  With one part, u = 2^-11, spectra whose values are all alike were off by up to 2.1 roundings."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod
from rows_util import EPS32, stored

pytestmark = pytest.mark.gpu

STEP = (3.4445, -4.7750, 2.0315)


def error_before_rounding(rows, cols, steps):
    grown = np.sqrt(sum(1.6 ** (2 * i) for i in range(steps)))
    return 2 * 5 * (2.0 ** -21 / np.sqrt(3) + EPS32 * np.sqrt(rows + cols)) * grown


def matrix(rows, cols, kind, seed=0):
    rng = np.random.default_rng(seed + rows + 3 * cols)
    side = min(rows, cols)
    few = max(1, side // 8)
    rank = lambda k: rng.normal(size=(rows, k)) @ rng.normal(size=(k, cols)) / np.sqrt(k)  # noqa: E731
    frame = lambda n, k: np.linalg.qr(rng.normal(size=(n, k)))[0]  # noqa: E731
    if kind == "full":
        return rng.normal(size=(rows, cols))
    if kind == "low":
        return rank(few)
    if kind == "mixed":
        return rank(few) + 0.3 * rng.normal(size=(rows, cols))
    if kind == "one":
        return rank(1)
    if kind == "spike":  # one element that is nearly all of it
        x = 1e-3 * rng.normal(size=(rows, cols))
        x[rows // 2, cols // 3] = side
        return x
    if kind == "decay":
        return (frame(rows, side) * np.logspace(0, -3, side)) @ frame(cols, side).T
    part = {"flat": side, "third": max(1, side // 3)}[kind]
    return frame(rows, part) @ frame(cols, part).T


@pytest.mark.parametrize("kind", ["full", "low", "mixed", "one", "spike", "decay", "flat", "third"])
@pytest.mark.parametrize("rows,cols,steps", [(24, 300, 4), (24, 300, 5), (83, 84, 5), (139, 139, 5), (141, 141, 5), (300, 260, 5), (150, 600, 5), (768, 192, 5), (256, 256, 6),
                                             (45, 118, 3), (1100, 700, 5)])
def test_bf16_results_are_off_by_their_rounding(rows, cols, steps, kind):
    torch = torch_mod()
    x = stored(1e-3 * matrix(rows, cols, kind), wl.BF16)
    t = torch.from_numpy(x).to(torch.bfloat16).cuda()
    y = torch.empty_like(t)
    d = B.make_orthogonal_desc(rows, cols, wl.BF16, 1, steps, STEP)
    n = B.orthogonalize_workspace_bytes(d)
    B.orthogonalize(d, t, y, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n)
    want = ro.newton_schulz(x, steps, STEP, 1e-7)
    off, least = np.linalg.norm(y.double().cpu().numpy() - want), np.linalg.norm(stored(want, wl.BF16) - want)
    assert off <= least + 2 * error_before_rounding(rows, cols, steps) * np.linalg.norm(want), off / least
    # (a tenth more at most where roundings of many elements make up the norm)
    assert kind == "spike" or off <= 1.1 * least, off / least


@pytest.mark.parametrize("batch,rows,cols", [(12, 3168, 24), (2, 38, 3475), (3, 2500, 60)])
def test_fp32_results_of_long_thin_matrices(batch, rows, cols):
    """The squares that X X^T adds up are all positive: a sum in order is off by half a rounding for each instruction's worth of them, half that in the mean, and the
    roundings of one sign add.  64 elements go to each of the two sums that one instruction in two adds to: K / 64 terms, K / 64 2^-26 of the element.  A step moves the singular values by
    (b s^2 + 2 c s^4) times that, 3 at most, and later steps turn its sign.  Parts of 22 bits and the short products leave 1e-6 besides."""
    torch = torch_mod()
    long = max(rows, cols)
    x = np.stack([stored(1e-3 * matrix(rows, cols, "mixed", i), wl.F32) for i in range(batch)])
    t = torch.from_numpy(x).float().cuda()
    y = torch.empty_like(t)
    d = B.make_orthogonal_desc(rows, cols, wl.F32, batch, 6, STEP)
    n = B.orthogonalize_workspace_bytes(d)
    B.orthogonalize(d, t, y, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n)
    want = np.stack([ro.newton_schulz(m, 6, STEP, 1e-7) for m in x])
    assert np.linalg.norm(y.double().cpu().numpy() - want) <= (3 * long / 64 * 2.0 ** -26 + 1e-6) * np.linalg.norm(want)
