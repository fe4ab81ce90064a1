"""Gradients of linear layers behind activations whose slopes the 16-bit types do not hold: no less exact than their own rounding lets them be.

A result w + e that is rounded once is off by the rounding of w + e, as large in the norm as that of w, and e.  The gradient at the sum is held in two parts, off by
2^-16 (bf16) and 2^-22 (fp16) of a term at most; slopes by some 30 roundings of fp32, 2^-19; sums of n terms by sqrt(n) roundings at random signs, 2^-18 for the
longest here.  Terms of random signs add these and the result alike, so e is below 2^-15 of the result in bf16 and 2^-17.5 in fp16: 2 % and 3 % of the rounding, whose norm
is 1.6e-3 and 2e-4 of the result.  Some hundred elements or more let two norms of roundings differ by 2 % more."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod
from rows_util import Rows, nan_vec, stored, torch_type

pytestmark = pytest.mark.gpu

ALLOWED = 1.05


def workspace(need):
    return torch_mod().full((max(need, 16),), 0xFF, dtype=torch_mod().uint8, device="cuda")


def gradients(x, w, z, g, dtype, act, start=0, want=("dx", "dw")):
    """-> dict of dx, dw, dbias as they come back, and the names of the products' forms."""
    torch = torch_mod()
    tt, nan = torch_type(dtype), float("nan")
    (rows, K), N = x.shape, len(w)
    pad = -K % 8
    X, W = Rows(rows, K, tt, K + pad, start, nan).set(x), Rows(N, K, tt, K + pad, start, nan).set(w)
    Z, G = Rows(rows, N, tt, N, start, nan).set(z), Rows(rows, N, tt, N, start, nan).set(g)
    DX, DW, DB = Rows(rows, K, tt, K + pad, start, 7.0), Rows(N, K, tt, K + pad, start, 7.0), nan_vec(N)
    d = B.make_linear_desc(rows, N, K, dtype, act, X.ld, W.ld, None, G.ld)
    need = B.linear_bwd_workspace_bytes(d)
    B.linear_bwd(d, X.ptr, W.ptr, Z.ptr, G.ptr, DX.ptr if "dx" in want else None, DW.ptr if "dw" in want else None, DB, workspace(need), need)
    torch.cuda.synchronize()
    assert DX.untouched(None if "dx" in want else 0) and DW.untouched(None if "dw" in want else 0)
    return {"dx": DX.host(), "dw": DW.host(), "dbias": DB.double().cpu().numpy()}, [B.linear_form(d, X.ptr, W.ptr, i) for i in (1, 2)]


def inputs(rows, N, K, dtype, seed=0):
    rng = np.random.default_rng(seed + rows + 7 * N + 13 * K)
    return (stored(rng.normal(size=(rows, K)), dtype), stored(rng.normal(size=(N, K)) * K ** -0.5, dtype), stored(1.5 * rng.normal(size=(rows, N)), dtype),
            stored(0.1 * rng.normal(size=(rows, N)), dtype))


def held_to_their_rounding(got, x, w, z, g, dtype, act, want=("dx", "dw")):
    ref = dict(zip(("dx", "dw", "dbias"), ro.linear_bwd(x, w, z, g, act)))
    for k in want:
        off, least = np.linalg.norm(got[k] - ref[k]), np.linalg.norm(stored(ref[k], dtype) - ref[k])
        assert off <= ALLOWED * least, "%s is off by %.3f times its rounding" % (k, off / least)
    assert np.linalg.norm(got["dbias"] - ref["dbias"]) <= 2.0 ** -17 * np.linalg.norm(np.abs(g).sum(0))


@pytest.mark.parametrize("dtype", [wl.F16, wl.BF16])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("rows,N,K,start", [(1, 64, 300, 0), (5, 100, 128, 1), (33, 48, 40, 0), (200, 1003, 999, 0), (777, 1283, 1001, 1), (300, 264, 136, 8), (3000, 100, 200, 0),
                                            (2048, 768, 192, 0)])
def test_gradients_are_off_by_their_own_rounding(rows, N, K, start, act, dtype):
    t = inputs(rows, N, K, dtype)
    held_to_their_rounding(gradients(*t, dtype, act, start)[0], *t, dtype, act)


# form -> which product, rows, N, K, elements the operands start at
FORMS = {
    "1 parts_tile64x64": (30, 40, 24, 0), "1 parts_tile64x64_any": (30, 40, 24, 1), "1 parts_tile128x128": (1000, 40, 1032, 0),
    "1 parts_tile128x128_any": (1000, 40, 1032, 1), "1 parts_tile192x192": (2000, 72, 2056, 0), "1 parts_tile256x256": (2600, 40, 4104, 0),
    "1 parts_tile256x256+parts_tile128x128": (4100, 40, 4104, 0), "1 parts_tile128x128_any+parts_tile64x64_any": (2000, 72, 2056, 1),
    "1 parts_tile64x64_split4": (40, 1000, 1032, 0), "1 parts_tile64x64_any_split7": (40, 2100, 2056, 1), "1 parts_tile128x128_split7": (72, 2056, 2056, 0),
    "1 parts_tile128x128_any_split7": (72, 2056, 2056, 1), "1 parts_tile192x192_split8": (40, 5000, 5000, 0), "1 parts_tile256x256_split8": (2048, 16384, 1024, 0),
    "2 parts_tile64x64": (30, 40, 24, 0), "2 parts_tile64x64_any": (30, 40, 24, 1), "2 parts_tile128x128": (40, 1000, 1032, 0),
    "2 parts_tile128x128_any": (1, 4104, 2056, 1), "2 parts_tile192x192": (1, 4104, 2056, 0), "2 parts_tile256x256": (40, 3080, 4104, 0),
    "2 parts_tile256x256+parts_tile128x128": (40, 4104, 4104, 0), "2 parts_tile128x128_any+parts_tile64x64_any": (72, 2056, 2056, 1),
    "2 parts_tile64x64_split8": (2000, 40, 1032, 0), "2 parts_tile64x64_any_split8": (2000, 40, 1032, 1), "2 parts_tile128x128_split13": (4100, 40, 4104, 0),
    "2 parts_tile128x128_any_split13": (4100, 8, 2056, 1), "2 parts_tile192x192_split8": (5000, 40, 5000, 0), "2 parts_tile256x256_split16": (16384, 1024, 1024, 0),
}


@pytest.mark.parametrize("dtype", [wl.F16, wl.BF16])
@pytest.mark.parametrize("name", FORMS)
def test_every_form_of_two_parts(name, dtype):
    rows, N, K, start = FORMS[name]
    which, form = name.split()
    want = ("dx",) if which == "1" else ("dw",)
    t = inputs(rows, N, K, dtype)
    got, forms = gradients(*t, dtype, "gelu", start, want)
    assert forms[int(which) - 1] == form
    held_to_their_rounding(got, *t, dtype, "gelu", want)


def test_fp16_gradients_at_the_sum_past_the_types_range():
    """dout times a slope above one passes fp16's largest number, times one near zero what fp16 can tell from zero; the results do neither."""
    rows, N, K = 40, 64, 24
    rng = np.random.default_rng(1)
    x = stored(rng.choice([-1.0, 1.0], (rows, K)) * 2.0 ** -12, wl.F16)
    # slopes 1.13 and -0.006: half of dz is 2^15.05; 2^-22.4 and 2^-28.4, which two parts hold to 2^-36
    for z, g, w, off in ((1.4, 60000.0, 2.0 ** -14, 2.0 ** -17), (-3.25, 2.0 ** -14, 60000.0, 2.0 ** -13), (-3.25, 2.0 ** -20, 60000.0, 2.0 ** -7)):
        t = (x if g > 1 else x * 2.0 ** 27, stored(w * rng.uniform(0.5, 1, (N, K)), wl.F16), stored(np.full((rows, N), z), wl.F16), stored(np.full((rows, N), g), wl.F16))
        if g > 1:
            assert (t[3] * ro.activation(t[2], "gelu")[1]).max() > 65520.0
        got, _ = gradients(*t, wl.F16, "gelu")
        for k, ref in zip(("dx", "dw"), ro.linear_bwd(*t, "gelu")):
            assert np.isfinite(got[k]).all()
            size = np.abs(ref).max()
            assert np.abs(got[k] - ref).max() <= (2.0 ** -11 + off) * size + 2.0 ** -25, k


@pytest.mark.parametrize("dtype", [wl.F16, wl.BF16])
def test_an_infinite_gradient_stays_one(dtype):
    rows, N, K = 20, 40, 24
    x, w, z, g = (np.abs(t) + 0.5 for t in inputs(rows, N, K, dtype))
    g[3, 5] = np.inf
    got, _ = gradients(*(stored(t, dtype) for t in (x, w, z, g)), dtype, "silu")
    assert np.isposinf(got["dx"][3]).all() and np.isposinf(got["dw"][5]).all() and np.isposinf(got["dbias"][5])
    assert np.isfinite(np.delete(got["dx"], 3, 0)).all() and np.isfinite(np.delete(got["dw"], 5, 0)).all()
    g[3, 5] = np.nan
    got, _ = gradients(*(stored(t, dtype) for t in (x, w, z, g)), dtype, "silu")
    assert np.isnan(got["dx"][3]).all() and np.isnan(got["dw"][5]).all() and np.isfinite(np.delete(got["dx"], 3, 0)).all()
