"""The operators on rows without a GPU: refusals of every entry point, empty calls, and the oracle against closed forms and
differences."""
import ctypes

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


NORM_BAD = [dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=1 << 30), dict(ldx=7), dict(ldy=7), dict(eps=-1.0),
            dict(eps=float("nan")), dict(eps=float("inf"))]


@pytest.mark.parametrize("change", NORM_BAD)
def test_norm_descriptors_that_are_refused(change):
    d = B.make_norm_desc(4, 8)
    for k, v in change.items():
        setattr(d, k, v)
    if change == dict(cols=1 << 30):
        d.ldx = d.ldy = 1 << 30
    assert status(B.layernorm_fwd, d, P, P, P, 2 * P, P, P, stream=0) == B.CONV_EINVAL
    assert status(B.layernorm_quant_fwd, d, P, P, P, 2 * P, P, stream=0) == B.CONV_EINVAL
    assert status(B.layernorm_bwd, d, P, 2 * P, P, P, P, 3 * P, P, P, P, 1 << 20, stream=0) == B.CONV_EINVAL
    assert B.layernorm_bwd_workspace_bytes(d) == 0


def test_norm_pointers_that_are_refused():
    d = B.make_norm_desc(4, 8, B.CONV_F32)
    assert status(B.layernorm_fwd, d, None, P, P, 2 * P, stream=0) == B.CONV_EINVAL
    assert status(B.layernorm_fwd, d, P, P, P, None, stream=0) == B.CONV_EINVAL
    assert status(B.layernorm_fwd, d, P, P, P, P, stream=0) == B.CONV_EINVAL                # in place
    assert status(B.layernorm_fwd, d, P + 2, P, P, 2 * P, stream=0) == B.CONV_EINVAL        # not on an element
    assert status(B.layernorm_fwd, d, P, P + 2, P, 2 * P, stream=0) == B.CONV_EINVAL
    assert status(B.layernorm_fwd, d, P, P, P, 2 * P, P + 1, stream=0) == B.CONV_EINVAL
    d.dtype = 3
    assert status(B.layernorm_fwd, d, P, P, P, 2 * P, stream=0) == B.CONV_EDTYPE
    assert status(B.layernorm_bwd, d, P, P, P, P, P, 2 * P, P, P, P, 1 << 20, stream=0) == B.CONV_EDTYPE
    d = B.make_norm_desc(4, 8, ldy=16)
    assert status(B.layernorm_quant_fwd, d, P, P, P, 2 * P + 8, P, stream=0) == B.CONV_EINVAL  # 8-bit rows start on 16 bytes
    assert status(B.layernorm_quant_fwd, d, P, P, P, 2 * P, None, stream=0) == B.CONV_EINVAL
    d.ldy = 24
    assert status(B.layernorm_quant_fwd, d, P, P, P, 2 * P, P, stream=0) == B.CONV_EINVAL
    assert B.lib().layernorm_fwd(None, P, P, P, 2 * P, P, P, None) == B.CONV_EINVAL
    assert B.lib().layernorm_bwd_workspace_bytes(None) == 0


def test_norm_bwd_arguments_that_are_refused():
    d = B.make_norm_desc(40, 8)
    ws = B.layernorm_bwd_workspace_bytes(d)
    assert ws > 0
    ok = dict(stream=0)
    assert status(B.layernorm_bwd, d, P, P, P, P, P, None, None, None, P, ws, **ok) == B.CONV_EINVAL      # nothing asked for
    assert status(B.layernorm_bwd, d, P, 2 * P, P, None, P, 3 * P, P, P, P, ws, **ok) == B.CONV_EINVAL
    assert status(B.layernorm_bwd, d, P, 2 * P, P, P, None, 3 * P, P, P, P, ws, **ok) == B.CONV_EINVAL
    assert status(B.layernorm_bwd, d, P, 2 * P, P, P, P, P, P, P, P, ws, **ok) == B.CONV_EINVAL           # dx over x
    assert status(B.layernorm_bwd, d, P, 2 * P, P, P, P, 3 * P, P, P, None, 0, **ok) == B.CONV_EWORKSPACE
    assert status(B.layernorm_bwd, d, P, 2 * P, P, P, P, 3 * P, P, P, P, ws - 1, **ok) == B.CONV_EWORKSPACE
    assert status(B.layernorm_bwd, d, P, 2 * P, P, P, P, 3 * P, P, P, P + 8, ws, **ok) == B.CONV_EINVAL
    d.ldx = 9
    assert status(B.layernorm_bwd, d, P, 2 * P, P, P, P, 2 * P, P, P, P, ws, **ok) == B.CONV_EINVAL       # dx over dy, other strides


@pytest.mark.parametrize("change", [dict(rows=-1), dict(cols=0), dict(ldx=7), dict(ldq=0), dict(ldq=24), dict(rows=1 << 31)])
def test_quantize_descriptors_that_are_refused(change):
    d = B.make_quant_desc(4, 8)
    for k, v in change.items():
        setattr(d, k, v)
    assert status(B.quantize_rows, d, P, 2 * P, P, stream=0) == B.CONV_EINVAL


def test_quantize_pointers_that_are_refused():
    d = B.make_quant_desc(4, 8, B.CONV_F16)
    for args in ((None, 2 * P, P), (P, None, P), (P, 2 * P, None), (P, P, P), (P + 1, 2 * P, P), (P, 2 * P + 4, P), (P, 2 * P, P + 2)):
        assert status(B.quantize_rows, d, *args, stream=0) == B.CONV_EINVAL, args
    d.dtype = -1
    assert status(B.quantize_rows, d, P, 2 * P, P, stream=0) == B.CONV_EDTYPE
    assert B.lib().quantize_rows(None, P, 2 * P, P, None) == B.CONV_EINVAL


@pytest.mark.parametrize("change", [dict(rows=-1), dict(rows=1 << 31), dict(N=0), dict(K=0), dict(K=1 << 17, lda=1 << 17, ldw=1 << 17), dict(lda=16),
                                    dict(ldw=16), dict(lda=40), dict(ldw=40), dict(ldo=9), dict(flags=2), dict(N=1 << 24, ldo=1 << 24)])
def test_int_linear_descriptors_that_are_refused(change):
    d = B.make_int_linear_desc(4, 10, 20)
    for k, v in change.items():
        setattr(d, k, v)
    assert status(B.int_linear_fwd, d, P, P, 2 * P, P, P, 3 * P, P, 1 << 20, stream=0) == B.CONV_EINVAL
    assert B.int_linear_workspace_bytes(d) == 0


def test_int_linear_pointers_that_are_refused():
    d = B.make_int_linear_desc(4, 10, 20, B.CONV_BF16)
    good = [P, P, 2 * P, P, P, 3 * P]
    for i, bad in ((0, None), (1, None), (2, None), (3, None), (5, None), (0, P + 8), (2, P + 8), (1, P + 2), (4, P + 2), (5, P + 1), (5, P), (5, 2 * P)):
        args = list(good)
        args[i] = bad
        assert status(B.int_linear_fwd, d, *args, P, 1 << 20, stream=0) == B.CONV_EINVAL, (i, bad)
    few = B.make_int_linear_desc(4, 10, 1 << 16)
    need = B.int_linear_workspace_bytes(few)
    assert need > 0
    assert status(B.int_linear_fwd, few, *good, None, 0, stream=0) == B.CONV_EWORKSPACE
    assert status(B.int_linear_fwd, few, *good, P, need - 1, stream=0) == B.CONV_EWORKSPACE
    assert status(B.int_linear_fwd, few, *good, P + 8, need, stream=0) == B.CONV_EINVAL
    d.dtype = 5
    assert status(B.int_linear_fwd, d, *good, P, 1 << 20, stream=0) == B.CONV_EDTYPE
    assert B.lib().int_linear_fwd(None, P, P, P, P, P, P, None, 0, None) == B.CONV_EINVAL


def test_int_linear_form_by_name():
    form = lambda rows, N, K, a=P, w=P, **kw: B.int_linear_form(B.make_int_linear_desc(rows, N, K, **kw), a, w)  # noqa: E731
    assert form(1, 4096, 4096) == "rows16" and form(3, 20, 30000) == "rows16_split16"
    assert form(4000, 4000, 2048) == "tile256x256"
    # rows that begin inside a line of 128 bytes, by their stride or by where they start
    assert form(1500, 1500, 256) == "tile128x128" == form(1500, 1500, 256, None, None)
    assert {form(1500, 1500, 256, P + 16), form(1500, 1500, 256, P, P + 48), form(1500, 1500, 256, lda=272)} == {"tile128x128_lines"}
    assert form(5, 70, 100, lda=1 << 23) == "any" and form(0, 8, 8) == ""
    # a workspace is asked for where the form's name says that a reduction is shared
    for size in ((3, 20, 30000), (130, 257, 16000), (1, 4096, 4096), (1500, 1500, 260)):
        assert (B.int_linear_workspace_bytes(B.make_int_linear_desc(*size)) > 0) == ("split" in form(*size))
    for bad in (dict(a=P + 8), dict(w=P + 8), dict(lda=40), dict(rows=-1)):
        with pytest.raises(B.ConvError):
            form(**{**dict(rows=4, N=8, K=16), **bad})


@pytest.mark.parametrize("change", [dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(ldx=99), dict(ldg=99), dict(top=-1), dict(top=65), dict(top=101)])
def test_logprob_descriptors_that_are_refused(change):
    d = B.make_logprob_desc(4, 100, top=5)
    for k, v in change.items():
        setattr(d, k, v)
    assert status(B.logprob_fwd, d, P, P, P, P, P, P, P, P, 1 << 20, stream=0) == B.CONV_EINVAL
    assert status(B.logprob_bwd, d, P, P, P, P, P, P, 2 * P, stream=0) == B.CONV_EINVAL
    assert B.logprob_workspace_bytes(d) == 0


def test_logprob_more_alternatives_than_columns():
    d = B.make_logprob_desc(4, 3, top=4)
    assert status(B.logprob_fwd, d, P, P, P, P, P, P, P, P, 1 << 20, stream=0) == B.CONV_EINVAL


def test_logprob_pointers_that_are_refused():
    d = B.make_logprob_desc(4, 100, B.CONV_F16, top=5)
    good = [P, P, P, P, P, P, P]  # logits target logp lse entropy top_id top_logp
    for i, bad in ((0, None), (1, None), (0, P + 1), (1, P + 4), (2, P + 2), (3, P + 1), (5, P + 4), (5, None), (6, None)):
        args = list(good)
        args[i] = bad
        assert status(B.logprob_fwd, d, *args, P, 1 << 20, stream=0) == B.CONV_EINVAL, (i, bad)
    assert status(B.logprob_fwd, d, P, P, None, None, None, None, None, P, 1 << 20, stream=0) == B.CONV_EINVAL  # nothing asked for
    good = [P, P, P, P, P, P, 2 * P]  # logits target lse entropy g_logp g_entropy dlogits
    for i, bad in ((0, None), (1, None), (2, None), (3, None), (6, None), (6, P + 1), (4, P + 2)):
        args = list(good)
        args[i] = bad
        assert status(B.logprob_bwd, d, *args, stream=0) == B.CONV_EINVAL, (i, bad)
    assert status(B.logprob_bwd, d, P, P, P, P, None, None, 2 * P, stream=0) == B.CONV_EINVAL
    d.ldg = 104
    assert status(B.logprob_bwd, d, P, P, P, P, P, P, P, stream=0) == B.CONV_EINVAL  # in place with other strides
    d.dtype = 9
    assert status(B.logprob_fwd, d, P, P, P, P, P, P, P, P, 1 << 20, stream=0) == B.CONV_EDTYPE
    assert B.lib().logprob_fwd(None, P, P, P, P, P, P, P, P, 0, None) == B.CONV_EINVAL
    assert B.lib().logprob_bwd(None, P, P, P, P, P, P, P, None) == B.CONV_EINVAL


def test_no_rows_is_a_valid_call_that_enqueues_nothing():
    assert status(B.layernorm_fwd, B.make_norm_desc(0, 8), None, None, None, None, stream=0) == B.CONV_OK
    assert status(B.layernorm_quant_fwd, B.make_norm_desc(0, 8, ldy=16), None, None, None, None, None, stream=0) == B.CONV_OK
    assert status(B.layernorm_bwd, B.make_norm_desc(0, 8), None, None, None, None, None, P, None, None, stream=0) == B.CONV_OK
    assert status(B.quantize_rows, B.make_quant_desc(0, 8), None, None, None, stream=0) == B.CONV_OK
    assert status(B.int_linear_fwd, B.make_int_linear_desc(0, 8, 8), None, None, None, None, None, None, stream=0) == B.CONV_OK
    assert status(B.logprob_fwd, B.make_logprob_desc(0, 8), None, None, None, stream=0) == B.CONV_OK
    assert status(B.logprob_bwd, B.make_logprob_desc(0, 8), None, P, None, None, P, None, None, stream=0) == B.CONV_OK


def test_descriptor_sizes_match_the_header():
    assert ctypes.sizeof(B.norm_desc) == 40 and ctypes.sizeof(B.quant_desc) == 32
    assert ctypes.sizeof(B.int_linear_desc) == 48 and ctypes.sizeof(B.logprob_desc) == 40


class Buffer:
    """What another library's array looks like to the binding."""

    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        if isinstance(self.address, Exception):
            raise self.address
        return self.address


def test_addresses_of_other_kinds_of_whole_numbers():
    d = B.make_norm_desc(4, 8)
    for address in (P, np.int64(P), np.uint64(P)):
        assert status(B.layernorm_fwd, d, Buffer(address), None, None, Buffer(address), stream=0) == B.CONV_EINVAL  # in place
    with pytest.raises(TypeError):
        B.layernorm_fwd(d, Buffer(None), None, None, Buffer(P), stream=0)
    with pytest.raises(AttributeError, match="gone"):
        B.layernorm_fwd(d, Buffer(AttributeError("gone")), None, None, Buffer(P), stream=0)
    for other in ("x", 1.5, np.zeros(3)):
        with pytest.raises(TypeError, match="expected a torch tensor"):
            B.layernorm_fwd(d, other, None, None, Buffer(P), stream=0)


# ---- the oracle ------------------------------------------------------------------------------------------------------


def test_oracle_layernorm_closed_forms_and_differences():
    rng = np.random.default_rng(1)
    y, mean, rstd = ro.layernorm(np.array([[1.0, 3.0]]), None, None, 0.0)
    assert np.allclose(y, [[-1, 1]]) and mean[0] == 2 and rstd[0] == 1
    x, dy = rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    gamma, beta = rng.normal(size=7), rng.normal(size=7)
    loss = lambda x, g, b: float((ro.layernorm(x, g, b, 1e-5)[0] * dy).sum())  # noqa: E731
    _, mean, rstd = ro.layernorm(x, gamma, beta, 1e-5)
    dx, dg, db = ro.layernorm_bwd(x, dy, gamma, mean, rstd)
    h = 1e-6
    for i in range(3):
        for j in range(7):
            e = np.zeros_like(x)
            e[i, j] = h
            assert abs((loss(x + e, gamma, beta) - loss(x - e, gamma, beta)) / (2 * h) - dx[i, j]) < 1e-7
    for j in range(7):
        e = np.zeros(7)
        e[j] = h
        assert abs((loss(x, gamma + e, beta) - loss(x, gamma - e, beta)) / (2 * h) - dg[j]) < 1e-7
        assert abs((loss(x, gamma, beta + e) - loss(x, gamma, beta - e)) / (2 * h) - db[j]) < 1e-7


def test_oracle_quantize_and_product():
    q, s = ro.quantize_rows(np.array([[127.0, -63.5, 0.49, 62.5], [0, 0, 0, 0], [1, np.nan, 2, 3]], dtype=np.float32))
    assert q[0].tolist() == [127, -64, 0, 62] and abs(s[0] - 1) < 1e-6
    assert q[1].tolist() == [0] * 4 and s[1] == np.float32(2.0 ** -126)
    assert q[2].tolist() == [0] * 4 and np.isnan(s[2])
    v, _ = ro.int_linear(np.array([[1, -2]], dtype=np.int8), np.array([2.0]), np.array([[3, 4], [5, -6]], dtype=np.int8), np.array([1.0, 0.5]), np.array([1.0, 0.0]), True)
    assert v.tolist() == [[0.0, 17.0]]


def test_oracle_logprob_closed_forms_and_differences():
    rng = np.random.default_rng(2)
    r = ro.logprob(np.zeros((1, 4)), np.array([2]), 3)
    assert np.isclose(r["logp"][0], -np.log(4)) and np.isclose(r["entropy"][0], np.log(4)) and r["top_id"][0].tolist() == [0, 1, 2]
    r = ro.logprob(np.array([[-np.inf, 0.0, -np.inf], [-np.inf] * 3, [0, np.nan, np.inf]]), np.array([0, 1, -1]), 2)
    assert r["logp"].tolist() == [-np.inf, -np.inf, 0.0] and r["entropy"][:2].tolist() == [0.0, 0.0] and np.isnan(r["entropy"][2])
    assert r["top_id"].tolist() == [[1, 0], [0, 1], [1, 2]]
    x, gl, gh = rng.normal(size=(2, 6)) * 2, rng.normal(size=2), rng.normal(size=2)
    target = np.array([3, -1])

    def loss(x):
        r = ro.logprob(x, target, 0)
        return float((r["logp"] * gl + r["entropy"] * gh).sum())

    r = ro.logprob(x, target, 0)
    dx = ro.logprob_bwd(x, target, r["lse"], r["entropy"], gl, gh)
    h = 1e-6
    for i in range(2):
        for j in range(6):
            e = np.zeros_like(x)
            e[i, j] = h
            assert abs((loss(x + e) - loss(x - e)) / (2 * h) - dx[i, j]) < 1e-7


def accepted(call, desc, nulls, **kw):
    """Whether an empty call with this descriptor is valid: the descriptor's checks come first."""
    return status(call, desc, *[None] * nulls, stream=0, **kw) == B.CONV_OK


def test_columns_and_strides_are_accepted_up_to_the_stated_limits():
    for ok, cols in ((True, (1 << 30) - 1), (False, 1 << 30)):
        for extra in (0, 1, 1 << 33):  # whatever the strides
            ld = (cols + 15) // 16 * 16 + 16 * extra
            assert accepted(B.layernorm_fwd, B.make_norm_desc(0, cols, ldx=ld, ldy=ld), 4) == ok, (cols, extra)
            assert accepted(B.layernorm_quant_fwd, B.make_norm_desc(0, cols, ldx=ld, ldy=ld), 5) == ok, (cols, extra)
            assert accepted(B.quantize_rows, B.make_quant_desc(0, cols, ldx=ld, ldq=ld), 3) == ok, (cols, extra)
            assert (B.layernorm_bwd_workspace_bytes(B.make_norm_desc(40, cols, ldx=ld, ldy=ld)) > 0) == ok, (cols, extra)
    for ok, cols in ((True, (1 << 31) - (1 << 20) - 1), (False, (1 << 31) - (1 << 20))):
        for ld in (cols, cols + 1, 1 << 33):
            assert accepted(B.logprob_fwd, B.make_logprob_desc(0, cols, ldx=ld, ldg=ld), 3) == ok, (cols, ld)
    assert accepted(B.int_linear_fwd, B.make_int_linear_desc(0, (1 << 24) - 1, (1 << 17) - 1, lda=1 << 33, ldw=1 << 33, ldo=1 << 33), 6)


@pytest.mark.parametrize("dtype,es", [(B.CONV_F32, 4), (B.CONV_BF16, 2)])
def test_tensors_whose_offsets_would_overflow_are_refused(dtype, es):
    """A tensor spans at most 2^62 bytes."""
    rows = (1 << 31) - 1
    ld = (1 << 62) // es // rows // 16 * 16
    assert B.layernorm_bwd_workspace_bytes(B.make_norm_desc(rows, 8, dtype, ldx=ld, ldy=ld)) > 0
    assert B.layernorm_bwd_workspace_bytes(B.make_norm_desc(rows, 8, dtype, ldx=ld + 16, ldy=8)) == 0
    assert B.layernorm_bwd_workspace_bytes(B.make_norm_desc(rows, 8, dtype, ldx=8, ldy=ld + 16)) == 0
    assert B.logprob_workspace_bytes(B.make_logprob_desc(1, 1 << 20, dtype, ldx=1 << 40, ldg=1 << 40)) > 0
    assert B.logprob_workspace_bytes(B.make_logprob_desc(2, 1 << 20, dtype, ldx=(1 << 61) // es + 1)) == 0
    assert B.logprob_workspace_bytes(B.make_logprob_desc(2, 1 << 20, dtype, ldg=(1 << 61) // es + 1)) == 0
    few = dict(rows=4, N=10, K=1 << 16, dtype=dtype)
    assert B.int_linear_workspace_bytes(B.make_int_linear_desc(**few, lda=1 << 40, ldw=1 << 40, ldo=1 << 40)) > 0
    for k, n in (("lda", 4), ("ldw", 10), ("ldo", 4 * es)):
        assert B.int_linear_workspace_bytes(B.make_int_linear_desc(**few, **{k: (1 << 62) // n // 16 * 16 + 16})) == 0
    for strides in (dict(ldx=ld + 16), dict(ldq=(1 << 62) // rows // 16 * 16 + 16)):
        assert status(B.quantize_rows, B.make_quant_desc(rows, 8, dtype, **strides), P, 2 * P, P, stream=0) == B.CONV_EINVAL
