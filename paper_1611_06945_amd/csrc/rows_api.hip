// C entry points of the operators on rows: layer norm, row quantiser, 8-bit product, log probabilities.  Arguments are
// checked before the first HIP call; the kernels' launchers choose among their forms.
#include <algorithm>
#include <climits>
#include <cmath>

#include "common.h"

using namespace convfwd;

namespace {

bool known(int dtype) { return dtype == CONV_F32 || dtype == CONV_F16 || dtype == CONV_BF16; }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
// a float vector: NULL allowed
bool vec_ok(const void* p) { return aligned(p, 4); }
constexpr int64_t kMostRows = INT32_MAX;
// A tensor spans at most 2^62 bytes, so that no offset in it, in elements or bytes, passes 63 bits.
bool spans(int64_t rows, int64_t stride, int size) { return stride <= ((int64_t)1 << 62) / size / std::max<int64_t>(rows, 1); }

int check_norm(const norm_desc* d)
{
    if (!d) return CONV_EINVAL;
    if (!known(d->dtype)) return CONV_EDTYPE;
    if (d->rows < 0 || d->rows > kMostRows || d->cols < 1 || d->cols >= (1 << 30)) return CONV_EINVAL;
    const int es = dtype_size(d->dtype);
    if (d->ldx < d->cols || d->ldy < d->cols || !spans(d->rows, d->ldx, es) || !spans(d->rows, d->ldy, es)) return CONV_EINVAL;
    if (!(d->eps >= 0.0f) || std::isinf(d->eps)) return CONV_EINVAL;
    return CONV_OK;
}

int check_logprob(const logprob_desc* d)
{
    if (!d) return CONV_EINVAL;
    if (!known(d->dtype)) return CONV_EDTYPE;
    if (d->rows < 0 || d->rows > kMostRows || d->cols < 1 || d->cols > INT32_MAX - (1 << 20)) return CONV_EINVAL;
    const int es = dtype_size(d->dtype);
    if (d->ldx < d->cols || d->ldg < d->cols || !spans(d->rows, d->ldx, es) || !spans(d->rows, d->ldg, es)) return CONV_EINVAL;
    if (d->top < 0 || d->top > 64 || d->top > d->cols) return CONV_EINVAL;
    return CONV_OK;
}

int check_int_linear(const int_linear_desc* d)
{
    if (!d) return CONV_EINVAL;
    if (!known(d->dtype)) return CONV_EDTYPE;
    if (d->rows < 0 || d->rows > kMostRows || d->N < 1 || d->K < 1 || d->K >= (1 << 17)) return CONV_EINVAL;
    if (d->N >= (1 << 24)) return CONV_EINVAL;  // tiles of one band of rows fit a launch
    if (d->lda < d->K || d->ldw < d->K || d->ldo < d->N || d->lda % 16 || d->ldw % 16) return CONV_EINVAL;
    if (!spans(d->rows, d->lda, 1) || !spans(d->N, d->ldw, 1) || !spans(d->rows, d->ldo, dtype_size(d->dtype))) return CONV_EINVAL;
    if (d->flags & ~(uint32_t)CONV_FLAG_RELU) return CONV_EINVAL;
    return CONV_OK;
}

// Runs a launcher; nothing it throws leaves the C interface.
template <typename F>
int guarded(const char* what, F launch) noexcept
{
    try {
        const hipError_t e = launch();
        return e == hipSuccess ? CONV_OK : hip_status(e, what);
    } catch (...) {
        return CONV_EHIP;
    }
}

}  // namespace

extern "C" {

int layernorm_fwd(const norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                  float* rstd, void* stream)
{
    const int rc = check_norm(desc);
    if (rc) return rc;
    if (!vec_ok(gamma) || !vec_ok(beta) || !vec_ok(mean) || !vec_ok(rstd)) return CONV_EINVAL;
    if (desc->rows == 0) return CONV_OK;
    const int es = dtype_size(desc->dtype);
    if (!x || !y || x == y || !aligned(x, es) || !aligned(y, es)) return CONV_EINVAL;
    NormArgs a = {};
    a.x = x, a.gamma = gamma, a.beta = beta, a.y = y, a.mean = mean, a.rstd = rstd;
    a.rows = desc->rows, a.ldx = desc->ldx, a.ldy = desc->ldy, a.cols = desc->cols, a.eps = desc->eps;
    return guarded("layernorm_fwd", [&] { return launch_layernorm_fwd(a, desc->dtype, (hipStream_t)stream); });
}

int layernorm_quant_fwd(const norm_desc* desc, const void* x, const float* gamma, const float* beta, int8_t* q, float* scale,
                        void* stream)
{
    const int rc = check_norm(desc);
    if (rc) return rc;
    if (desc->ldy % 16 || !vec_ok(gamma) || !vec_ok(beta) || !vec_ok(scale)) return CONV_EINVAL;
    if (desc->rows == 0) return CONV_OK;
    if (!x || !q || !scale || (const void*)q == x || !aligned(x, dtype_size(desc->dtype)) || !aligned(q, 16)) return CONV_EINVAL;
    NormArgs a = {};
    a.x = x, a.gamma = gamma, a.beta = beta, a.q = q, a.scale = scale;
    a.rows = desc->rows, a.ldx = desc->ldx, a.ldy = desc->ldy, a.cols = desc->cols, a.eps = desc->eps;
    return guarded("layernorm_quant_fwd", [&] { return launch_layernorm_fwd(a, desc->dtype, (hipStream_t)stream); });
}

size_t layernorm_bwd_workspace_bytes(const norm_desc* desc)
{
    return check_norm(desc) ? 0 : layernorm_bwd_workspace(desc->rows, desc->cols, desc->dtype);
}

int layernorm_bwd(const norm_desc* desc, const void* x, const void* dy, const float* gamma, const float* mean, const float* rstd,
                  void* dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_norm(desc);
    if (rc) return rc;
    if (!vec_ok(gamma) || !vec_ok(mean) || !vec_ok(rstd) || !vec_ok(dgamma) || !vec_ok(dbeta)) return CONV_EINVAL;
    if (!dx && !dgamma && !dbeta) return CONV_EINVAL;
    const int es = dtype_size(desc->dtype);
    if (desc->rows > 0) {
        if (!x || !dy || !mean || !rstd || !aligned(x, es) || !aligned(dy, es) || !aligned(dx, es)) return CONV_EINVAL;
        if (dx == x || (dx == dy && desc->ldx != desc->ldy)) return CONV_EINVAL;
    }
    if (dgamma || dbeta) {
        const size_t need = layernorm_bwd_workspace(desc->rows, desc->cols, desc->dtype);
        if (need && (!workspace || workspace_bytes < need)) return CONV_EWORKSPACE;
        if (!aligned(workspace, 16)) return CONV_EINVAL;
    } else if (desc->rows == 0) {
        return CONV_OK;
    }
    NormArgs a = {};
    a.x = x, a.dy = dy, a.gamma = gamma, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
    a.dx = dx, a.dgamma = dgamma, a.dbeta = dbeta, a.ws = (float*)workspace;
    a.rows = desc->rows, a.ldx = desc->ldx, a.ldy = desc->ldy, a.cols = desc->cols, a.eps = desc->eps;
    return guarded("layernorm_bwd", [&] { return launch_layernorm_bwd(a, desc->dtype, (hipStream_t)stream); });
}

int quantize_rows(const quant_desc* desc, const void* x, int8_t* q, float* scale, void* stream)
{
    if (!desc) return CONV_EINVAL;
    if (!known(desc->dtype)) return CONV_EDTYPE;
    if (desc->rows < 0 || desc->rows > kMostRows || desc->cols < 1 || desc->cols >= (1 << 30)) return CONV_EINVAL;
    if (desc->ldx < desc->cols || desc->ldq < desc->cols || desc->ldq % 16) return CONV_EINVAL;
    if (!spans(desc->rows, desc->ldx, dtype_size(desc->dtype)) || !spans(desc->rows, desc->ldq, 1)) return CONV_EINVAL;
    if (desc->rows == 0) return CONV_OK;
    if (!x || !q || !scale || (const void*)q == x || !aligned(x, dtype_size(desc->dtype)) || !aligned(q, 16) || !vec_ok(scale)) return CONV_EINVAL;
    QuantArgs a = {x, q, scale, desc->rows, desc->ldx, desc->ldq, desc->cols};
    return guarded("quantize_rows", [&] { return launch_quantize_rows(a, desc->dtype, (hipStream_t)stream); });
}

size_t int_linear_workspace_bytes(const int_linear_desc* desc)
{
    return check_int_linear(desc) ? 0 : int_linear_workspace(desc->rows, desc->N, desc->K);
}

int int_linear_form(const int_linear_desc* desc, const int8_t* a, const int8_t* w, char* buf, size_t n)
{
    const int rc = check_int_linear(desc);
    if (rc) return rc;
    if (!buf || n == 0 || !aligned(a, 16) || !aligned(w, 16)) return CONV_EINVAL;
    buf[0] = 0;
    if (desc->rows == 0) return CONV_OK;
    IntLinearArgs g = {};
    g.a = a, g.w = w, g.rows = desc->rows, g.lda = desc->lda, g.ldw = desc->ldw, g.ldo = desc->ldo, g.N = desc->N, g.K = desc->K;
    int_linear_form_name(g, buf, n);
    return CONV_OK;
}

int int_linear_fwd(const int_linear_desc* desc, const int8_t* a, const float* a_scale, const int8_t* w, const float* w_scale,
                   const float* bias, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_int_linear(desc);
    if (rc) return rc;
    if (desc->rows == 0) return CONV_OK;
    if (!a || !a_scale || !w || !w_scale || !out) return CONV_EINVAL;
    if (!aligned(a, 16) || !aligned(w, 16) || !vec_ok(a_scale) || !vec_ok(w_scale) || !vec_ok(bias)) return CONV_EINVAL;
    if (!aligned(out, dtype_size(desc->dtype)) || out == (const void*)a || out == (const void*)w) return CONV_EINVAL;
    const size_t need = int_linear_workspace(desc->rows, desc->N, desc->K);
    if (need && (!workspace || workspace_bytes < need)) return CONV_EWORKSPACE;
    if (!aligned(workspace, 16)) return CONV_EINVAL;
    IntLinearArgs g = {a, a_scale, w, w_scale, bias, out, (int*)workspace, desc->rows, desc->lda, desc->ldw, desc->ldo,
                       desc->N, desc->K, (desc->flags & CONV_FLAG_RELU) ? 1 : 0};
    return guarded("int_linear_fwd", [&] { return launch_int_linear(g, desc->dtype, (hipStream_t)stream); });
}

size_t logprob_workspace_bytes(const logprob_desc* desc)
{
    return check_logprob(desc) ? 0 : logprob_workspace(desc->rows, desc->cols, desc->top, desc->dtype);
}

int logprob_fwd(const logprob_desc* desc, const void* logits, const int64_t* target, float* logp, float* lse, float* entropy,
                int64_t* top_id, float* top_logp, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_logprob(desc);
    if (rc) return rc;
    if (!vec_ok(logp) || !vec_ok(lse) || !vec_ok(entropy) || !vec_ok(top_logp) || !aligned(top_id, 8) || !aligned(target, 8)) return CONV_EINVAL;
    if ((top_id == nullptr) != (top_logp == nullptr)) return CONV_EINVAL;
    if (desc->rows == 0) return CONV_OK;
    const bool top = top_id && desc->top > 0;
    if (!logits || !aligned(logits, dtype_size(desc->dtype)) || (logp && !target)) return CONV_EINVAL;
    if (!logp && !lse && !entropy && !top) return CONV_EINVAL;
    const size_t need = logprob_workspace(desc->rows, desc->cols, desc->top, desc->dtype);
    if (need && (!workspace || workspace_bytes < need)) return CONV_EWORKSPACE;
    if (!aligned(workspace, 16)) return CONV_EINVAL;
    LogprobArgs a = {};
    a.x = logits, a.target = target, a.logp = logp, a.lse = lse, a.entropy = entropy;
    a.top_id = top ? top_id : nullptr, a.top_logp = top ? top_logp : nullptr, a.ws = workspace;
    a.rows = desc->rows, a.ldx = desc->ldx, a.ldg = desc->ldg, a.cols = desc->cols, a.top = top ? desc->top : 0;
    return guarded("logprob_fwd", [&] { return launch_logprob_fwd(a, desc->dtype, (hipStream_t)stream); });
}

int logprob_bwd(const logprob_desc* desc, const void* logits, const int64_t* target, const float* lse, const float* entropy,
                const float* g_logp, const float* g_entropy, void* dlogits, void* stream)
{
    const int rc = check_logprob(desc);
    if (rc) return rc;
    if (!vec_ok(lse) || !vec_ok(entropy) || !vec_ok(g_logp) || !vec_ok(g_entropy) || !aligned(target, 8)) return CONV_EINVAL;
    if ((!g_logp && !g_entropy) || (g_logp && !target) || (g_entropy && !entropy)) return CONV_EINVAL;
    if (desc->rows == 0) return CONV_OK;
    const int es = dtype_size(desc->dtype);
    if (!logits || !lse || !dlogits || !aligned(logits, es) || !aligned(dlogits, es)) return CONV_EINVAL;
    if (logits == dlogits && desc->ldx != desc->ldg) return CONV_EINVAL;
    LogprobArgs a = {};
    a.x = logits, a.target = target, a.lse = const_cast<float*>(lse), a.entropy = const_cast<float*>(entropy);
    a.g_logp = g_logp, a.g_entropy = g_entropy, a.dx = dlogits;
    a.rows = desc->rows, a.ldx = desc->ldx, a.ldg = desc->ldg, a.cols = desc->cols;
    return guarded("logprob_bwd", [&] { return launch_logprob_bwd(a, desc->dtype, (hipStream_t)stream); });
}

}  // extern "C"
