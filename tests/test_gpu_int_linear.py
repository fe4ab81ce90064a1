"""The product in 8-bit integers on the GPU: sums are exact, so only the scaling, the bias and the rounding are held to bounds."""
import numpy as np
import pytest

from oracle import rows_oracle as ro
from paper_1611_06945_amd import binding as B
from paper_1611_06945_amd import workloads as wl

from gpu_util import torch_mod
from rows_util import EPS32, ROUND, TINY, Rows, assert_close, torch_type, vec

pytestmark = pytest.mark.gpu

DTYPES = [wl.F32, wl.F16, wl.BF16]


def check(rows, N, K, dtype, relu=False, bias=True, pad=0, ldo=None, start=0, seed=0, extreme=False, nan_row=None):
    torch = torch_mod()
    rng = np.random.default_rng(seed + rows + 7 * N + 13 * K)
    lo, hi = (-128, -128) if extreme else (-128, 127)
    a, w = rng.integers(lo, hi + 1, size=(rows, K)).astype(np.int8), rng.integers(lo, hi + 1, size=(N, K)).astype(np.int8)
    sa, sw = rng.uniform(0.5, 2, rows).astype(np.float32) / 1000, rng.uniform(0.5, 2, N).astype(np.float32) / 1000
    if nan_row is not None:
        sa[nan_row] = np.nan
    b = rng.normal(size=N).astype(np.float32) if bias else None
    # what lies behind the columns is read up to the next 16 bytes: its values must not matter
    A = Rows(rows, K, torch.int8, B.row_stride(K) + pad, fill=77).set(a)
    W = Rows(N, K, torch.int8, B.row_stride(K) + 2 * pad, fill=-55).set(w)
    Y = Rows(rows, N, torch_type(dtype), ldo, start, fill=7.0)
    d = B.make_int_linear_desc(rows, N, K, dtype, relu, A.ld, W.ld, Y.ld)
    need = B.int_linear_workspace_bytes(d)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    B.int_linear_fwd(d, A.ptr, vec(sa), W.ptr, vec(sw), None if b is None else vec(b), Y.ptr, ws, need)
    torch.cuda.synchronize()
    v, size = ro.int_linear(a, sa, w, sw, b, relu)
    if nan_row is not None:
        v[nan_row] = np.nan
    tol = 5 * EPS32 * size
    assert_close(Y.host(), v, tol + ROUND[dtype] * (np.abs(v) + tol) + TINY[dtype], "out")
    assert Y.untouched()
    return Y


ROWS = [1, 2, 3, 7, 8, 15, 16, 17, 31, 33, 63, 65, 100, 129]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("N,K", [(1, 1), (10, 17), (16, 64), (33, 63), (100, 128), (130, 65), (257, 300), (64, 1001)])
def test_small_products(rows, N, K):
    check(rows, N, K, DTYPES[(rows + N) % 3], relu=bool(N % 2), bias=bool(K % 2), pad=16 * (rows % 3), seed=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,K", [(1, 4096, 4096), (1, 1000, 16384), (5, 4096, 9216), (20, 1000, 4096), (16, 16, 16384), (32, 513, 2050), (64, 2048, 1024),
                                      (200, 1003, 999), (777, 1283, 1001), (256, 256, 128), (257, 255, 129), (512, 512, 512), (1000, 128, 4096), (129, 3000, 384),
                                      (1024, 1024, 256), (1300, 1111, 640), (2048, 768, 1600)])
def test_products(rows, N, K, dtype):
    check(rows, N, K, dtype, relu=rows % 2 == 0, seed=2)


@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("rows,N,K", [(1, 10, 40000), (3, 7, 65001), (20, 30, 30000), (64, 100, 16384), (33, 17, 13001), (128, 128, 12000), (100, 1, 100003)])
def test_reductions_that_workgroups_share(rows, N, K, relu):
    assert B.int_linear_workspace_bytes(B.make_int_linear_desc(rows, N, K)) > 0
    check(rows, N, K, DTYPES[K % 3], relu=relu, pad=32, ldo=N + 3, start=1, seed=7)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,N,ldo,start", [(3, 50, 53, 1), (40, 130, 131, 3), (300, 300, 311, 5), (300, 260, 264, 1), (600, 512, 520, 0), (17, 1001, 1002, 2)])
def test_outputs_that_are_slices(rows, N, ldo, start, dtype):
    check(rows, N, 200, dtype, ldo=ldo, start=start, pad=48, seed=3)


@pytest.mark.parametrize("a_start,w_start", [(0, 0), (16, 0), (48, 112), (96, 80)])
@pytest.mark.parametrize("pad", [0, 16, 48, 112])
@pytest.mark.parametrize("rows,N,K", [(70, 70, 1), (64, 300, 128), (130, 1000, 129), (600, 900, 300), (260, 1500, 500), (1500, 1500, 260), (600, 513, 1040)])
def test_rows_that_begin_anywhere_in_a_line(rows, N, K, pad, a_start, w_start):
    torch = torch_mod()
    rng = np.random.default_rng(rows + N + K + pad)
    a, w = rng.integers(-128, 128, size=(rows, K)).astype(np.int8), rng.integers(-128, 128, size=(N, K)).astype(np.int8)
    A = Rows(rows, K, torch.int8, B.row_stride(K) + pad, a_start, fill=-99).set(a)
    W = Rows(N, K, torch.int8, B.row_stride(K) + 3 * pad, w_start, fill=101).set(w)
    one_a, one_w = np.full(rows, 2.0 ** -3, np.float32), np.full(N, 2.0, np.float32)
    Y = Rows(rows, N, torch.float32, N + 1, 1, fill=7.0)
    d = B.make_int_linear_desc(rows, N, K, wl.F32, False, A.ld, W.ld, Y.ld)
    need = B.int_linear_workspace_bytes(d)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    B.int_linear_fwd(d, A.ptr, vec(one_a), W.ptr, vec(one_w), None, Y.ptr, ws, need)
    torch.cuda.synchronize()
    # sums below 2^24 in steps of a quarter: exact
    assert np.array_equal(Y.host(), (a.astype(np.float64) @ w.astype(np.float64).T) / 4)
    assert Y.untouched()


@pytest.mark.parametrize("dtype", [wl.F16, wl.BF16])
@pytest.mark.parametrize("rows,N,K,ldo,start", [(600, 900, 300, 901, 0), (600, 901, 300, 904, 3), (260, 4097, 200, 4097, 0), (1500, 1511, 260, 1511, 5),
                                                (3000, 1537, 130, 1537, 1), (3001, 1543, 128, 1544, 7), (4000, 4001, 2000, 4001, 0), (600, 833, 300, 835, 2)])
def test_odd_row_lengths(rows, N, K, ldo, start, dtype):
    check(rows, N, K, dtype, ldo=ldo, start=start, relu=bool(N % 4 == 1), seed=8)


@pytest.mark.parametrize("rows", [1, 20, 300])
def test_the_largest_sums(rows):
    check(rows, 40, (1 << 17) - 1, wl.F32, extreme=True, seed=4)


@pytest.mark.parametrize("rows", [3, 40, 300])
@pytest.mark.parametrize("relu", [False, True])
def test_a_row_whose_scale_is_nan_is_nan(rows, relu):
    check(rows, 70, 100, wl.F16, relu=relu, nan_row=rows - 1, seed=5)


@pytest.mark.parametrize("rows", [1, 18, 130, 700])
def test_the_same_call_gives_the_same_bits(rows):
    a, b = (check(rows, 300, 2000, wl.F32, seed=6).host() for _ in range(2))
    assert np.array_equal(a, b)


@pytest.mark.parametrize("rows", [65535 * 16 + 37, 65535 * 64 + 37])
def test_more_rows_than_one_launch_holds(rows):
    """65535 tiles of rows are one launch's; a narrow product over more of them against the sums by hand."""
    torch = torch_mod()
    N, K = 3, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    a = torch.randint(-128, 128, (rows, K), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    one_a, one_w = torch.ones(rows, device="cuda"), torch.ones(N, device="cuda")
    out = torch.full((rows, N), float("nan"), device="cuda")
    d = B.make_int_linear_desc(rows, N, K)
    need = B.int_linear_workspace_bytes(d)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    B.int_linear_fwd(d, a, one_a, w, one_w, None, out, ws, need)
    want = (a.float()[:, None, :] * w.float()[None]).sum(2)
    assert bool((out == want).all())


def test_operands_beyond_four_gigabytes():
    """Rows whose offsets pass 32 bits, in the 8-bit operand and in the output."""
    torch = torch_mod()
    rows, N, K, lda, ldo = 600, 130, 96, 1 << 23, 1 << 22   # 5.0e9 bytes of a, 1.0e10 bytes of an fp32 output
    a = torch.zeros(rows * lda, dtype=torch.int8, device="cuda").view(rows, lda)
    a[:, :K] = torch.randint(-128, 128, (rows, K), device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (N, K), device="cuda", dtype=torch.int8)
    out = torch.zeros(rows * ldo, device="cuda").view(rows, ldo)
    d = B.make_int_linear_desc(rows, N, K, wl.F32, lda=lda, ldo=ldo)
    need = B.int_linear_workspace_bytes(d)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    B.int_linear_fwd(d, a, torch.ones(rows, device="cuda"), w, torch.ones(N, device="cuda"), None, out, ws, need)
    want = a[:, :K].contiguous().float() @ w.float().t().contiguous()
    assert bool((out[:, :N] == want).all()) and bool((out[:, N:N + 64] == 0).all())


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("rows,N,K", [(40, 9000, 500), (300, 1100, 1300), (900, 1300, 1000), (1100, 4000, 2100), (2100, 4000, 1000), (4200, 4300, 1100), (8300, 500, 260),
                                      (300, 20000, 130)])
def test_products_of_every_form(rows, N, K, dtype):
    """Sums small enough to be whole numbers in the output type are compared bit for bit; each case is another form's."""
    torch = torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    lim = 120 if dtype == wl.F32 else 1
    A = torch.randint(-lim, lim + 1, (rows, B.row_stride(K) + 16), generator=g, device="cuda", dtype=torch.int8)
    W = torch.randint(-lim, lim + 1, (N, B.row_stride(K)), generator=g, device="cuda", dtype=torch.int8)
    sa = torch.randint(1, 3, (rows,), generator=g, device="cuda").float()
    sw = torch.randint(1, 3, (N,), generator=g, device="cuda").float()
    out = torch.full((rows, N), float("nan"), device="cuda", dtype=torch_type(dtype))
    d = B.make_int_linear_desc(rows, N, K, dtype, lda=A.shape[1], ldw=W.shape[1])
    need = B.int_linear_workspace_bytes(d)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    B.int_linear_fwd(d, A, sa, W, sw, None, out, ws, need)
    want = (A[:, :K].double() @ W[:, :K].double().t().contiguous()) * sa.double()[:, None] * sw.double()[None, :]
    assert bool((out.double() == want.to(out.dtype).double()).all())


def exact_product(rows, N, K, dtype, lda, ldw, ldo, start=0, relu=False, a_start=0, splits=None):
    """Whole-number scales and biases and codes small enough that every sum is a whole number below 2^24: bit for bit, whatever the
    form, with what lies around the output untouched.  Returns the form's name."""
    torch = torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + N + K)
    lim = 50 if dtype == wl.F32 else 1
    assert lim * lim * K ** 0.5 * 4 * 8 < 1 << 24  # eight standard deviations and more

    def codes(n, ld, start):
        flat = torch.empty(start + n * ld, dtype=torch.int8, device="cuda")
        view = flat[start:].view(n, ld)
        view[:, :B.row_stride(K)] = torch.randint(-128, 128, (n, B.row_stride(K)), generator=g, device="cuda", dtype=torch.int8)
        view[:, :K] = torch.randint(-lim, lim + 1, (n, K), generator=g, device="cuda", dtype=torch.int8)
        return view

    A, W = codes(rows, lda, a_start), codes(N, ldw, 0)
    sa, sw = (torch.randint(1, 3, (n,), generator=g, device="cuda").float() for n in (rows, N))
    bias = torch.randint(-9, 10, (N,), generator=g, device="cuda").float()
    Y = Rows(rows, N, torch_type(dtype), ldo, start, fill=7.0)
    d = B.make_int_linear_desc(rows, N, K, dtype, relu, lda, ldw, ldo)
    need = B.int_linear_workspace_bytes(d)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    B.int_linear_fwd(d, A, sa, W, sw, bias, Y.ptr, ws, need)
    want = (A[:, :K].double() @ W[:, :K].double().t().contiguous()) * sa.double()[:, None] * sw.double()[None, :] + bias.double()
    want = torch.relu(want) if relu else want
    assert torch.equal(Y.view.double(), want.to(Y.view.dtype).double())
    assert Y.untouched()
    return B.int_linear_form(d, A, W)


# rows, channels, reduction, strides of the codes past the next 16 bytes, the form that takes them
FORMS = [(9, 300, 700, 0, "rows16"), (3, 20, 30000, 16, "rows16_split16"), (20, 1000, 4096, 0, "rows32"), (30, 100, 20000, 48, "rows32_split16"),
         (60, 500, 2000, 16, "rows64"), (130, 257, 16000, 0, "rows64_split5"), (260, 1500, 512, 0, "tile64x64"), (600, 900, 300, 16, "tile64x64_lines"),
         (900, 1300, 1024, 0, "tile64x128"), (900, 1300, 1000, 16, "tile64x128_lines"), (1500, 1500, 256, 0, "tile128x128"), (1500, 1500, 260, 80, "tile128x128_lines"),
         (2100, 4000, 1024, 0, "tile128x128_two_a_cu"), (2100, 4001, 1000, 16, "tile128x128_two_a_cu"), (4000, 4000, 2048, 0, "tile256x256"),
         (4001, 4003, 2000, 32, "tile256x256"), (5, 70, 100, (1 << 23) - 112, "any")]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("rows,N,K,pad,form", FORMS)
def test_each_form_with_each_way_out(rows, N, K, pad, form, odd, dtype):
    """Every form, in every output type, with rows of outputs that begin on words and with rows that do not."""
    ldo = N + (N % 2 == 0) if odd else (N + 8) // 8 * 8
    assert exact_product(rows, N, K, dtype, B.row_stride(K) + pad, B.row_stride(K) + 2 * pad if form != "any" else B.row_stride(K), ldo, int(odd), relu=odd) == form


@pytest.mark.parametrize("rows,N,K,less,form", [(64, 64, 100, 16, "rows64"), (257, 700, 100, 16, "tile64x64_lines"), (257, 700, 100, 128, "tile64x64"),
                                                (700, 1500, 100, 16, "tile64x128_lines"), (1500, 1500, 100, 16, "tile128x128_lines"),
                                                (1500, 1500, 100, 128, "tile128x128"), (1500, 3000, 100, 48, "tile128x128_two_a_cu"), (3000, 3000, 4000, 16, "tile256x256")])
def test_tiles_of_the_longest_strides(rows, N, K, less, form):
    """Row strides just below the 2^23 from which on another kernel takes the product: the largest offsets within a tile."""
    torch = torch_mod()
    ld = (1 << 23) - less
    assert torch.cuda.mem_get_info()[0] > (rows + N) * ld + (8 << 30)
    assert exact_product(rows, N, K, wl.F32, ld, ld, N) == form
    torch.cuda.empty_cache()
