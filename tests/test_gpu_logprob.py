"""Log probabilities, entropy, alternatives and their gradient on the GPU against the 64-bit oracle.

Bounds: a sum of exponentials formed by threads and joined as a tree is off by (terms of a thread + joins) units of 2^-24,
an exponential of d by a few units and |d| more (its argument is rounded): with N = 128 + cols / 64 units for the sums,
lse is off by N + average |d| units plus its own roundings, the entropy by N (1 + average |d|) + average d^2."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod
from rows_util import EPS32, ROUND, TINY, Rows, assert_close, nan_vec, stored, torch_type, vec

pytestmark = pytest.mark.gpu

DTYPES = [wl.F32, wl.F16, wl.BF16]
SHAPES = [(1, 1), (3, 2), (4, 10), (5, 63), (2, 64), (7, 100), (33, 257), (300, 17), (20, 1000), (3, 1024), (2, 4099), (1, 8192), (5, 20011), (1, 50257), (2, 131072), (1, 200003)]


def bounds(x, r):
    n = 128 + x.shape[1] / 64.0
    with np.errstate(invalid="ignore"):
        d = np.where(np.isfinite(x), x - np.where(np.isfinite(r["lse"]), r["lse"], 0)[:, None], 0.0)
        p = np.where(np.isfinite(x), np.exp(np.minimum(d, 0)), 0.0)
    big = np.where(np.isfinite(x), np.abs(x), 0).max(1)
    ad, ad2 = (p * np.abs(d)).sum(1), (p * d * d).sum(1)
    ls = np.where(np.isfinite(r["lse"]), np.abs(r["lse"]), 0)
    e_lse = EPS32 * (n + 4 * ad + 4 * (ls + big) + 16)
    spread = ad + np.log(x.shape[1])   # |d| is taken from the largest logit or from lse: they are log cols apart at most
    e_h = EPS32 * 4 * (n * (1 + spread) + ad2 + spread ** 2 + 16)
    return e_lse, e_h, big


def forward(x, dtype, target, top, ld=None, start=0, want=31):
    torch = torch_mod()
    rows, cols = x.shape
    X = Rows(rows, cols, torch_type(dtype), ld, start, fill=float("nan")).set(x)
    d = B.make_logprob_desc(rows, cols, dtype, top, X.ld)
    need = B.logprob_workspace_bytes(d)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    logp, lse, h = nan_vec(rows), nan_vec(rows), nan_vec(rows)
    ids = torch.full((rows, max(top, 1)), -7, dtype=torch.int64, device="cuda")
    lps = torch.full((rows, max(top, 1)), float("nan"), device="cuda")
    t = None if target is None else torch.from_numpy(np.asarray(target, dtype=np.int64)).cuda()
    B.logprob_fwd(d, X.ptr, t, logp if want & 1 else None, lse if want & 2 else None, h if want & 4 else None,
                  ids if want & 8 else None, lps if want & 8 else None, ws, need)
    torch.cuda.synchronize()
    return X, [v.cpu().numpy() for v in (logp, lse, h, ids[:, :top], lps[:, :top])]


def check(x, dtype, target, top, ld=None, start=0, want=31):
    X, (logp, lse, h, ids, lps) = forward(x, dtype, target, top, ld, start, want)
    r = ro.logprob(x, target, top)
    e_lse, e_h, big = bounds(x, r)
    if want & 1:
        assert_close(logp, r["logp"], e_lse + 2 * EPS32 * (big + np.where(np.isfinite(r["logp"]), np.abs(r["logp"]), 0)), "logp")
    if want & 2:
        assert_close(lse, r["lse"], e_lse, "lse")
    if want & 4:
        assert_close(h, r["entropy"], e_h, "entropy")
    if want & 8 and top:
        assert np.array_equal(ids, r["top_id"]), "alternatives"
        assert_close(lps, r["top_logp"], (e_lse + 4 * EPS32 * (big + np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0))))[:, None], "top_logp")
    return X, r


def logits(rows, cols, dtype, seed, sigma=2.5):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, sigma, size=(rows, cols))
    x[np.arange(rows), rng.integers(0, cols, rows)] += 4
    return stored(x, dtype), rng.integers(0, cols, rows)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_logprob_fwd(rows, cols, dtype):
    x, t = logits(rows, cols, dtype, rows + cols)
    for top in sorted({0, min(1, cols), min(5, cols), min(20, cols)}):
        check(x, dtype, t, top)


@pytest.mark.parametrize("cols", [64, 65, 1000, 30000])
@pytest.mark.parametrize("top", [2, 16, 33, 63, 64])
def test_many_alternatives(cols, top):
    x, t = logits(4, cols, wl.F16, cols + top)
    check(x, wl.F16, t, top)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,ld,start", [(100, 101, 1), (1000, 1003, 3), (5003, 5007, 5), (40001, 40010, 7)])
def test_rows_that_start_anywhere(cols, ld, start, dtype):
    x, t = logits(6, cols, dtype, cols)
    check(x, dtype, t, 5, ld, start)


@pytest.mark.parametrize("rows,cols", [(300, 1000), (70, 20000), (1025, 501), (4100, 40)])
def test_many_rows(rows, cols):
    x, t = logits(rows, cols, wl.BF16, rows)
    check(x, wl.BF16, t, 3)


@pytest.mark.parametrize("want", [1, 2, 4, 8, 3, 6, 14, 9])
def test_some_outputs_only(want):
    x, t = logits(5, 777, wl.F32, want)
    check(x, wl.F32, t if want & 1 else None, 4, want=want) if want & 1 else check_without_target(x, want)


def check_without_target(x, want):
    _, (logp, lse, h, ids, lps) = forward(x, wl.F32, None, 4, want=want)
    r = ro.logprob(x, None, 4)
    e_lse, e_h, big = bounds(x, r)
    assert np.isnan(logp).all()
    if want & 2:
        assert_close(lse, r["lse"], e_lse, "lse")
    if want & 4:
        assert_close(h, r["entropy"], e_h, "entropy")
    if want & 8:
        assert np.array_equal(ids, r["top_id"])


@pytest.mark.parametrize("cols", [3, 70, 1000, 9000, 100000])
def test_masks_empty_rows_ties_and_values_that_are_not_finite(cols):
    rng = np.random.default_rng(cols)
    low = -65504.0   # the lowest fp16 value, as masks use it
    top = min(cols, 20)
    x, t = logits(16, cols, wl.F16, cols)
    x[0][rng.random(cols) < 0.5] = -np.inf
    x[1] = -np.inf                                  # nothing is left
    x[2] = -np.inf
    x[2, cols - 1] = 1.0                            # one is left, the last
    x[3] = low                                      # masked with the lowest value throughout
    x[4][rng.random(cols) < 0.9] = low
    x[5] = 2.0                                      # all equal: the lowest indices
    x[6] = np.round(x[6])                           # many ties
    x[7, cols // 2] = np.nan
    x[8, cols // 3] = np.inf
    x[9] = np.where(np.arange(cols) % 2, -0.0, 0.0)  # zeros of both signs are equal
    x[10] = np.sort(x[10])
    x[11] = np.sort(x[11])[::-1]
    x[12] = np.where(np.arange(cols) < cols // 2, -np.inf, x[12])
    x[13] = np.where(np.arange(cols) < (cols + 1) // 2, x[13], -np.inf)
    x[14] = np.nan
    x[15, :] = -np.inf
    x[15, 0] = np.nan
    t[2], t[5] = cols - 1, 0
    t[0], t[10] = -1, -100
    t[6] = cols                                     # no such column
    check(x, wl.F16, t, top)
    check(x, wl.F16, t, min(cols, 64))


@pytest.mark.parametrize("cols", [2000, 70000])
def test_alternatives_that_crowd_together(cols):
    """All large values next to each other, or a fixed distance apart: whatever shares the row among threads gets them unevenly."""
    rng = np.random.default_rng(cols)
    x, t = logits(12, cols, wl.F32, cols)
    for i, step in enumerate((1, 2, 4, 8, 16, 64, 256, 512, 1024)):
        at = (np.arange(200) * step + 5 * i) % cols
        x[i, at] = 20 + rng.normal(size=at.size)
    x[9, 100:1500] = 9.0
    x[10] = np.arange(cols)[::-1] * 1e-3
    x[11] = np.arange(cols) * 1e-3
    check(stored(x, wl.F32), wl.F32, t, 20)
    check(stored(x, wl.F32), wl.F32, t, 64)


@pytest.mark.parametrize("big", [80.0, 1e4, 1e30])
def test_large_logits(big):
    x, t = logits(4, 3000, wl.F32, 5)
    check(stored(x * big, wl.F32), wl.F32, t, 5)


# ---- the gradient ----------------------------------------------------------------------------------------------------


def check_bwd(x, dtype, t, gl, gh, ld=None, ldg=None, start=0, in_place=False):
    torch = torch_mod()
    rows, cols = x.shape
    r = ro.logprob(x, t, 0)
    lse, h = r["lse"].astype(np.float32), r["entropy"].astype(np.float32)
    X = Rows(rows, cols, torch_type(dtype), ld, start, fill=float("nan")).set(x)
    G = X if in_place else Rows(rows, cols, torch_type(dtype), ldg, start, fill=7.0)
    d = B.make_logprob_desc(rows, cols, dtype, 0, X.ld, G.ld)
    B.logprob_bwd(d, X.ptr, None if t is None else torch.from_numpy(np.asarray(t, dtype=np.int64)).cuda(), vec(lse), vec(h),
                  None if gl is None else vec(gl), None if gh is None else vec(gh), G.ptr)
    torch.cuda.synchronize()
    l64, h64 = lse.astype(np.float64), h.astype(np.float64)
    want = ro.logprob_bwd(x, t, l64, h64, gl, gh)
    with np.errstate(invalid="ignore", over="ignore"):
        fine = np.isfinite(x) & np.isfinite(l64)[:, None]
        lp = np.where(fine, x - np.where(np.isfinite(l64), l64, 0)[:, None], 0)
        p = np.where(fine, np.exp(lp), 0)
        e_lp = 2 * EPS32 * np.where(fine, np.abs(x) + np.abs(l64)[:, None], 0)   # of x - lse, and of its use
        e_p = p * (e_lp + EPS32 * (2 * np.abs(lp) + 8)) + 2.0 ** -126   # an exponential below the normal numbers may be 0
        hh = np.where(np.isfinite(h64), np.abs(h64), 0)[:, None]
        g1 = np.abs(np.nan_to_num(gl))[:, None] if gl is not None else 0.0
        g2 = np.abs(gh)[:, None] if gh is not None else 0.0
        tol = g1 * (e_p + 4 * EPS32 * (1.0 * (np.arange(cols) == (-1 if t is None else np.asarray(t)[:, None])) + p))
        tol = tol + g2 * (e_p * (np.abs(lp) + hh) + p * e_lp + 6 * EPS32 * p * (np.abs(lp) + hh))
    if not in_place:
        assert G.untouched()
    assert_close(G.host(), want, tol * 1.02 + ROUND[dtype] * (np.abs(np.nan_to_num(want)) + tol) + TINY[dtype] + 2.0 ** -126, "dlogits")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_logprob_bwd(rows, cols, dtype):
    x, t = logits(rows, cols, dtype, rows + 3 * cols)
    rng = np.random.default_rng(cols)
    gl, gh = (rng.normal(size=rows).astype(np.float32).astype(np.float64) for _ in range(2))
    check_bwd(x, dtype, t, gl, gh)
    check_bwd(x, dtype, t, gl, None)
    check_bwd(x, dtype, None, None, gh)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,ld,ldg,start", [(100, 101, 107, 1), (1000, 1003, 1003, 3), (5003, 5007, 5003, 5), (64, 64, 65, 0)])
def test_logprob_bwd_of_slices(cols, ld, ldg, start, dtype):
    x, t = logits(6, cols, dtype, cols)
    gl = np.full(6, -0.25)
    check_bwd(x, dtype, t, gl, gl * 2, ld, ldg, start)
    check_bwd(x, dtype, t, gl, gl * 2, ld, ld, start, in_place=True)


@pytest.mark.parametrize("cols", [5, 900, 60000])
def test_logprob_bwd_of_masks_and_empty_rows(cols):
    x, t = logits(8, cols, wl.BF16, cols)
    rng = np.random.default_rng(1)
    x[0][rng.random(cols) < 0.5] = -np.inf
    x[1] = -np.inf
    x[2] = -np.inf
    x[2, 3] = 1.0
    x[3, 1] = np.nan
    t[4] = -1
    t[5] = cols
    x[6] = stored(np.full(cols, -3.3e38), wl.BF16)
    gl, gh = rng.normal(size=8).astype(np.float32).astype(np.float64), rng.normal(size=8).astype(np.float32).astype(np.float64)
    check_bwd(x, wl.BF16, t, gl, gh)
    check_bwd(x, wl.BF16, t, gl, None)


def test_logprob_bwd_agrees_with_differences():
    rows, cols, h = 4, 501, 1e-5
    x, t = logits(rows, cols, wl.F32, 77)
    rng = np.random.default_rng(3)
    v, gl, gh = rng.normal(size=(rows, cols)), rng.normal(size=rows).astype(np.float32), rng.normal(size=rows).astype(np.float32)
    X, (logp, lse, ent, _, _) = forward(x, wl.F32, t, 0)
    G = Rows(rows, cols, torch_type(wl.F32))
    B.logprob_bwd(B.make_logprob_desc(rows, cols), X.ptr, torch_mod().from_numpy(t).cuda(), vec(lse), vec(ent), vec(gl), vec(gh), G.ptr)

    def f(x):
        r = ro.logprob(x, t, 0)
        return r["logp"] * gl + r["entropy"] * gh

    want = (f(x + h * v) - f(x - h * v)) / (2 * h)
    assert np.allclose((G.host() * v).sum(1), want, atol=1e-4, rtol=1e-4)


def test_offsets_beyond_32_bits():
    """Rows of a tensor of 2.2e9 logits: forward and gradient of the last ones against the same rows on their own."""
    torch = torch_mod()
    rows, cols, ld = 20, 5000, 110_000_000
    free, _ = torch.cuda.mem_get_info()
    assert free > 12 * 2 ** 30
    x = torch.zeros(rows * ld, dtype=torch.float16, device="cuda").view(rows, ld)
    x[:, :cols] = torch.randn(rows, cols, device="cuda") * 3
    own = x[:, :cols].contiguous()
    t = torch.randint(0, cols, (rows,), device="cuda")
    got = []
    for z, l in ((x, ld), (own, cols)):
        d = B.make_logprob_desc(rows, cols, wl.F16, 5, l, l)
        ws = torch.empty(max(16, B.logprob_workspace_bytes(d)), dtype=torch.uint8, device="cuda")
        o = [torch.empty(rows, device="cuda") for _ in range(3)] + [torch.empty(rows, 5, dtype=torch.int64, device="cuda"), torch.empty(rows, 5, device="cuda")]
        B.logprob_fwd(d, z, t, *o, ws, ws.numel())
        B.logprob_bwd(d, z, t, o[1], o[2], torch.ones(rows, device="cuda"), torch.ones(rows, device="cuda"), z)
        got.append(o + [z[:, :cols].contiguous()])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_more_rows_than_workgroups():
    torch = torch_mod()
    rows, cols, top = 300_001, 9, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.randint(-3, 4, (rows, cols), generator=g, device="cuda").float()
    t = torch.randint(0, cols, (rows,), generator=g, device="cuda")
    d = B.make_logprob_desc(rows, cols, wl.F32, top)
    o = [torch.empty(rows, device="cuda") for _ in range(3)] + [torch.empty(rows, top, dtype=torch.int64, device="cuda"), torch.empty(rows, top, device="cuda")]
    B.logprob_fwd(d, x, t, *o, None, 0)
    lse = torch.logsumexp(x.double(), 1)
    assert torch.allclose(o[1].double(), lse, atol=1e-5, rtol=1e-5)
    assert torch.allclose(o[0].double(), x.double().gather(1, t[:, None])[:, 0] - lse, atol=1e-5, rtol=1e-5)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(o[3], order)
    dx = torch.empty_like(x)
    B.logprob_bwd(d, x, t, o[1], None, torch.ones(rows, device="cuda"), None, dx)
    want = -torch.exp(x.double() - o[1].double()[:, None])
    want.scatter_add_(1, t[:, None], torch.ones(rows, 1, dtype=torch.float64, device="cuda"))
    assert torch.allclose(dx.double(), want, atol=1e-5)


def test_gradient_of_a_row_of_more_columns_than_a_launch_holds():
    """A launch has 65535 runs of 1024 pieces of a row; the gradient of a longer one, against the formula in 64 bits by slices."""
    torch = torch_mod()
    cols = 65535 * 1024 * 4 + 4099
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(1, cols, generator=g, device="cuda")
    lse, target = torch.logsumexp(x.double(), 1).float(), torch.tensor([cols - 3], device="cuda")
    entropy, gl, gh = torch.full((1,), 3.0, device="cuda"), torch.full((1,), -1.5, device="cuda"), torch.full((1,), 0.5, device="cuda")
    dx = torch.full_like(x, float("nan"))
    B.logprob_bwd(B.make_logprob_desc(1, cols), x, target, lse, entropy, gl, gh, dx)
    ends = sorted({0, 1 << 20, cols // 2, 65535 * 1024 * 4 - 1024, cols - 4099 - 5000, cols - 4099, cols - 1500, cols})
    assert bool(torch.isfinite(dx).all())
    for j0, j1 in zip(ends, ends[1:]):
        j1 = min(j1, j0 + (1 << 24))
        lp = x[0, j0:j1].double() - lse.double()
        p = torch.exp(lp)
        want = -p * (-1.5 + 0.5 * (lp + 3.0))
        if j0 <= cols - 3 < j1:
            want[cols - 3 - j0] += -1.5
        # |lp| below 32, in units of 2^-24: x - lse is off by 16, its product with log2 e by 22 and by 7 for the constant, which the
        # exponential passes on, with two of its own; the factor and the products by a few
        size = p * (1.5 + 0.5 * (lp.abs() + 3.0))
        off = (dx[0, j0:j1].double() - want).abs()
        assert bool((off <= 2.0 ** -24 * (64 * size + 2 * want.abs() + 4 * (want.abs() > 1))).all()), (j0, j1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gh", [1e19, -1e25, 1e36])
def test_gradient_of_masked_columns_is_zero_however_large_that_of_the_entropy(dtype, gh):
    """p log p is 0 where p is 0; with a scaled loss the factor of p there must not overflow."""
    torch = torch_mod()
    rng = np.random.default_rng(3)
    x = stored(rng.normal(size=(3, 77)), dtype)
    x[:, 5::7] = -np.inf
    x[1, 6::7] = stored(np.array([-6e4]), dtype)[0]
    x[2, :] = -np.inf
    x[2, 9] = 0.0
    lse, h = (ro.logprob(x, None, 0)[k] for k in ("lse", "entropy"))
    X = Rows(3, 77, torch_type(dtype)).set(x)
    out = torch.full((3, 77), float("nan"), device="cuda", dtype=torch_type(dtype))
    B.logprob_bwd(B.make_logprob_desc(3, 77, dtype), X.ptr, None, vec(lse), vec(h), None, vec(np.full(3, gh)), out)
    got = out.double().cpu().numpy()
    p = np.exp(x - lse[:, None])
    assert (got[p == 0] == 0).all()
    assert not np.isnan(got).any()
    if dtype == wl.F32:
        # (the entropy as rounded to fp32: off by 2^-24 of itself)
        h32, l32 = h.astype(np.float32).astype(np.float64), lse.astype(np.float32).astype(np.float64)
        want = ro.logprob_bwd(x, None, l32, h32, None, np.full(3, gh))
        lp = np.where(p > 0, x - l32[:, None], 0.0)
        assert (np.abs(got - want) <= EPS32 * 16 * (1 + np.abs(lp)) * abs(gh) * p * (np.abs(lp) + h32[:, None] + 1)).all()


@pytest.mark.parametrize("cols", [5, 1000, 70001])
def test_log_probabilities_do_not_depend_on_where_the_logits_lie(cols):
    """Rows around a large value, and of the lowest value only: log probabilities are those of the differences to the largest logit,
    with the bounds of logits around 0."""
    rng = np.random.default_rng(cols)
    for dtype, rows in ((wl.F16, [np.full(cols, -65504.0), 32768 + 32.0 * rng.integers(-1, 2, cols), -60000.0 - 32 * rng.integers(0, 2, cols)]),
                        (wl.BF16, [np.full(cols, -(2.0 - 2.0 ** -7) * 2.0 ** 127), 2.0 ** 10 + 8 * rng.integers(-1, 2, cols), np.full(cols, 1e30)]),
                        (wl.F32, [np.full(cols, -(2.0 - 2.0 ** -23) * 2.0 ** 127), 1e7 + rng.integers(-5, 6, cols), -1e5 - rng.integers(0, 900, cols) / 128])):
        x = stored(np.stack(rows), dtype)
        t = rng.integers(0, cols, 3)
        _, (logp, _, h, ids, lps) = forward(x, dtype, t, 3)
        shifted = x - x.max(1, keepdims=True)  # exact in 64 bits
        r = ro.logprob(shifted, t, 3)
        e_lse, e_h, _ = bounds(shifted, r)
        assert_close(logp, r["logp"], e_lse + 2 * EPS32 * np.abs(r["logp"]), "logp")
        assert_close(lps, r["top_logp"], (e_lse + 4 * EPS32 * np.abs(r["lse"]))[:, None], "top_logp")
        assert_close(h, r["entropy"], e_h, "entropy")
        assert np.array_equal(ids, r["top_id"])
