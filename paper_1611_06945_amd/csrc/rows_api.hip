// C entry points of the operators on rows: layer norm, row quantiser, 8-bit product, log probabilities, linear layers, the norms around a
// block, Newton-Schulz steps.  Arguments are
// checked before the first HIP call; the kernels' launchers choose among their forms.
#include <algorithm>
#include <climits>
#include <cmath>
#include <initializer_list>

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

int check_linear(const linear_desc* d)
{
    if (!d) return CONV_EINVAL;
    if (!known(d->dtype)) return CONV_EDTYPE;
    if (d->rows < 0 || d->rows > kMostRows || d->N < 1 || d->K < 1 || d->N >= (1 << 24) || d->K >= (1 << 24)) return CONV_EINVAL;
    const int es = dtype_size(d->dtype);
    if (d->ldx < d->K || d->ldw < d->K || d->ldr < d->N || d->ldo < d->N) return CONV_EINVAL;
    if (!spans(d->rows, d->ldx, es) || !spans(d->N, d->ldw, es) || !spans(d->rows, d->ldr, es) || !spans(d->rows, d->ldo, es)) return CONV_EINVAL;
    const uint32_t act = d->flags & (CONV_FLAG_RELU | LINEAR_FLAG_GELU | LINEAR_FLAG_SILU);
    if (d->flags != act || (act & (act - 1))) return CONV_EINVAL;
    return CONV_OK;
}

LinearArgs linear_args(const linear_desc* d)
{
    LinearArgs a = {};
    a.rows = d->rows, a.ldx = d->ldx, a.ldw = d->ldw, a.ldr = d->ldr, a.ldo = d->ldo, a.N = d->N, a.K = d->K;
    a.act = d->flags & CONV_FLAG_RELU ? 1 : d->flags & LINEAR_FLAG_GELU ? 2 : d->flags & LINEAR_FLAG_SILU ? 3 : 0;
    return a;
}

int check_residual_norm(const residual_norm_desc* d)
{
    if (!d) return CONV_EINVAL;
    if (!known(d->dtype)) return CONV_EDTYPE;
    if (d->rows < 0 || d->rows > kMostRows || d->cols < 1 || d->cols >= (1 << 27) || d->gate_rows < 0) return CONV_EINVAL;
    const int es = dtype_size(d->dtype);
    for (const int64_t ld : {d->ldr, d->ldh, d->ldy})
        if (ld < d->cols || !spans(d->rows, ld, es)) return CONV_EINVAL;
    if (d->gate_rows && (d->ldg < d->cols || !spans(d->rows, d->ldg, es))) return CONV_EINVAL;
    if (!(d->eps >= 0.0f) || std::isinf(d->eps)) return CONV_EINVAL;
    if (d->flags & ~(RESIDUAL_NORM_RMS | RESIDUAL_NORM_POST | RESIDUAL_NORM_SIGMOID)) return CONV_EINVAL;
    return CONV_OK;
}

ResidualNormArgs residual_norm_args(const residual_norm_desc* d)
{
    ResidualNormArgs a = {};
    a.rows = d->rows, a.ldr = d->ldr, a.ldh = d->ldh, a.ldg = d->ldg, a.ldy = d->ldy, a.gate_rows = d->gate_rows, a.cols = d->cols, a.eps = d->eps;
    a.rms = (d->flags & RESIDUAL_NORM_RMS) != 0, a.post = (d->flags & RESIDUAL_NORM_POST) != 0, a.sigmoid = (d->flags & RESIDUAL_NORM_SIGMOID) != 0;
    return a;
}

int check_orthogonal(const orthogonal_desc* d)
{
    if (!d) return CONV_EINVAL;
    if (!known(d->dtype)) return CONV_EDTYPE;
    if (d->batch < 0 || d->batch > kMostRows || d->rows < 1 || d->cols < 1 || d->rows > (1 << 20) || d->cols > (1 << 20)) return CONV_EINVAL;
    if (std::min(d->rows, d->cols) > (1 << 17)) return CONV_EINVAL;
    if (d->steps < 1 || d->steps > 100 || d->ldx < d->cols || d->ldo < d->cols || d->stride_x < 0 || d->stride_o < 0) return CONV_EINVAL;
    const int es = dtype_size(d->dtype);
    if (!spans(d->rows, d->ldx, es) || !spans(d->rows, d->ldo, es) || !spans(d->batch, d->stride_x, es) || !spans(d->batch, d->stride_o, es)) return CONV_EINVAL;
    if (d->batch > 1 && d->stride_o < d->rows * d->ldo) return CONV_EINVAL;
    if (!std::isfinite(d->a) || !std::isfinite(d->b) || !std::isfinite(d->c) || !(d->eps >= 0.0f) || std::isinf(d->eps)) return CONV_EINVAL;
    // the workspace of a batch, too, is below 2^62 bytes
    const double side = std::min(d->rows, d->cols);
    if ((double)d->batch * (20.0 * d->rows * (d->cols + 64.0) + 16.0 * side * (side + 64.0)) > 0x1p61) return CONV_EINVAL;
    return CONV_OK;
}

OrthogonalArgs orthogonal_args(const orthogonal_desc* d)
{
    OrthogonalArgs a = {};
    a.batch = d->batch, a.rows = d->rows, a.cols = d->cols, a.ldx = d->ldx, a.ldo = d->ldo, a.stride_x = d->stride_x, a.stride_o = d->stride_o;
    a.steps = d->steps, a.a = d->a, a.b = d->b, a.c = d->c, a.eps = d->eps;
    return a;
}

// Whether an output is one of the inputs, or another output.
bool overlaps(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs)
{
    for (auto o = outputs.begin(); o != outputs.end(); ++o) {
        if (!*o) continue;
        for (const void* i : inputs)
            if (*o == i) return true;
        for (auto p = outputs.begin(); p != o; ++p)
            if (*o == *p) return true;
    }
    return false;
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

size_t linear_workspace_bytes(const linear_desc* desc)
{
    return check_linear(desc) ? 0 : linear_fwd_workspace(desc->rows, desc->N, desc->K, desc->dtype);
}

int linear_fwd(const linear_desc* desc, const void* x, const void* w, const float* bias, const void* residual, void* out, void* pre,
               void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_linear(desc);
    if (rc) return rc;
    if (desc->rows == 0) return CONV_OK;
    const int es = dtype_size(desc->dtype);
    if (!x || !w || !out || !aligned(x, es) || !aligned(w, es) || !aligned(out, es) || !aligned(residual, es) || !aligned(pre, es) || !vec_ok(bias)) return CONV_EINVAL;
    if (overlaps({out, pre}, {x, w, bias}) || (pre && pre == residual) || (residual == out && desc->ldr != desc->ldo)) return CONV_EINVAL;
    const size_t need = linear_fwd_workspace(desc->rows, desc->N, desc->K, desc->dtype);
    if (need && (!workspace || workspace_bytes < need)) return CONV_EWORKSPACE;
    if (!aligned(workspace, 16)) return CONV_EINVAL;
    LinearArgs a = linear_args(desc);
    a.x = x, a.w = w, a.bias = bias, a.residual = residual, a.out = out, a.pre = pre, a.ws = workspace;
    return guarded("linear_fwd", [&] { return launch_linear_fwd(a, desc->dtype, (hipStream_t)stream); });
}

size_t linear_bwd_workspace_bytes(const linear_desc* desc)
{
    return check_linear(desc) ? 0 : linear_bwd_workspace(desc->rows, desc->N, desc->K, linear_args(desc).act, desc->dtype);
}

int linear_bwd(const linear_desc* desc, const void* x, const void* w, const void* pre, const void* dout, void* dx, void* dw, float* dbias,
               void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_linear(desc);
    if (rc) return rc;
    const int es = dtype_size(desc->dtype);
    LinearArgs a = linear_args(desc);
    if (!dx && !dw && !dbias) return CONV_EINVAL;
    if (!aligned(x, es) || !aligned(w, es) || !aligned(pre, es) || !aligned(dout, es) || !aligned(dx, es) || !aligned(dw, es) || !vec_ok(dbias)) return CONV_EINVAL;
    if (desc->rows > 0) {
        if (!dout || (dw && !x) || (dx && !w) || (a.act && !pre)) return CONV_EINVAL;
        if (overlaps({dx, dw, dbias}, {x, w, pre, dout})) return CONV_EINVAL;
        const size_t need = linear_bwd_workspace(desc->rows, desc->N, desc->K, linear_args(desc).act, desc->dtype);
        if (need && (!workspace || workspace_bytes < need)) return CONV_EWORKSPACE;
        if (!aligned(workspace, 16)) return CONV_EINVAL;
    }
    a.x = x, a.w = w, a.pre_in = pre, a.dout = dout, a.dx = dx, a.dw = dw, a.dbias = dbias, a.ws = workspace;
    return guarded("linear_bwd", [&] { return launch_linear_bwd(a, desc->dtype, (hipStream_t)stream); });
}

int linear_form(const linear_desc* desc, const void* x, const void* w, int which, char* buf, size_t n)
{
    const int rc = check_linear(desc);
    if (rc) return rc;
    if (!buf || n == 0 || which < 0 || which > 2) return CONV_EINVAL;
    buf[0] = 0;
    if (desc->rows == 0) return CONV_OK;
    LinearArgs a = linear_args(desc);
    a.x = x, a.w = w;
    linear_form_name(a, desc->dtype, which, buf, n);
    return CONV_OK;
}

int residual_norm_fwd(const residual_norm_desc* desc, const void* r, const void* h, const void* gate, const float* gamma_h, const float* beta_h,
                      const float* scale, const float* gamma, const float* beta, void* r_out, void* y, float* stats, void* stream)
{
    const int rc = check_residual_norm(desc);
    if (rc) return rc;
    ResidualNormArgs a = residual_norm_args(desc);
    const int es = dtype_size(desc->dtype);
    for (const float* v : {gamma_h, beta_h, scale, gamma, beta})
        if (!vec_ok(v)) return CONV_EINVAL;
    if (!aligned(r, es) || !aligned(h, es) || !aligned(gate, es) || !aligned(r_out, es) || !aligned(y, es) || !aligned(stats, 16)) return CONV_EINVAL;
    if (!a.post && (gamma_h || beta_h)) return CONV_EINVAL;
    if (desc->rows == 0) return CONV_OK;
    if (!r || !h || !r_out || (gate != nullptr) != (desc->gate_rows > 0)) return CONV_EINVAL;
    if (overlaps({r_out, y, stats}, {h, gate, gamma_h, beta_h, scale, gamma, beta}) || y == r || (const void*)stats == r) return CONV_EINVAL;
    a.r = r, a.h = h, a.gate = gate, a.gamma_h = gamma_h, a.beta_h = beta_h, a.scale = scale, a.gamma = gamma, a.beta = beta;
    a.r_out = r_out, a.y = y, a.stats_out = stats;
    return guarded("residual_norm_fwd", [&] { return launch_residual_norm_fwd(a, desc->dtype, (hipStream_t)stream); });
}

size_t residual_norm_bwd_workspace_bytes(const residual_norm_desc* desc)
{
    return check_residual_norm(desc) ? 0 : residual_norm_bwd_workspace(desc->rows, desc->cols, desc->gate_rows, desc->dtype);
}

int residual_norm_bwd(const residual_norm_desc* desc, const void* r_out, const void* h, const void* gate, const float* gamma_h, const float* beta_h,
                      const float* scale, const float* gamma, const float* stats, const void* dr_out, const void* dy, void* dr, void* dh, void* dgate,
                      float* dgamma_h, float* dbeta_h, float* dscale, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_residual_norm(desc);
    if (rc) return rc;
    ResidualNormArgs a = residual_norm_args(desc);
    const int es = dtype_size(desc->dtype);
    for (const float* v : {gamma_h, beta_h, scale, gamma, (const float*)dgamma_h, (const float*)dbeta_h, (const float*)dscale, (const float*)dgamma, (const float*)dbeta})
        if (!vec_ok(v)) return CONV_EINVAL;
    for (const void* p : {r_out, h, gate, dr_out, dy, (const void*)dr, (const void*)dh, (const void*)dgate})
        if (!aligned(p, es)) return CONV_EINVAL;
    if (!aligned(stats, 16) || !aligned(workspace, 16)) return CONV_EINVAL;
    if (!dr && !dh && !dgate && !dgamma_h && !dbeta_h && !dscale && !dgamma && !dbeta) return CONV_EINVAL;
    if (!a.post && (gamma_h || beta_h || dgamma_h || dbeta_h)) return CONV_EINVAL;
    if (desc->rows > 0) {
        if (!h || (!dr_out && !dy) || (dy && !r_out) || ((dy || a.post) && !stats)) return CONV_EINVAL;
        if ((gate != nullptr) != (desc->gate_rows > 0) || (dgate && !gate)) return CONV_EINVAL;
        if (overlaps({dr, dh, dgate, dgamma_h, dbeta_h, dscale, dgamma, dbeta}, {r_out, h, gate, gamma_h, beta_h, scale, gamma, stats, dr_out, dy})) return CONV_EINVAL;
    }
    const size_t need = residual_norm_bwd_workspace(desc->rows, desc->cols, desc->gate_rows, desc->dtype);
    if (need && (!workspace || workspace_bytes < need)) return CONV_EWORKSPACE;
    a.x = r_out, a.h = h, a.gate = gate, a.gamma_h = gamma_h, a.beta_h = beta_h, a.scale = scale, a.gamma = gamma, a.stats = stats;
    a.dr_out = dr_out, a.dy = dy, a.dr = dr, a.dh = dh, a.dgate = dgate;
    a.dgamma_h = dgamma_h, a.dbeta_h = dbeta_h, a.dscale = dscale, a.dgamma = dgamma, a.dbeta = dbeta, a.ws = workspace;
    return guarded("residual_norm_bwd", [&] { return launch_residual_norm_bwd(a, desc->dtype, (hipStream_t)stream); });
}

size_t orthogonalize_workspace_bytes(const orthogonal_desc* desc)
{
    return check_orthogonal(desc) ? 0 : orthogonal_workspace(orthogonal_args(desc), desc->dtype);
}

int orthogonalize(const orthogonal_desc* desc, const void* x, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_orthogonal(desc);
    if (rc) return rc;
    if (desc->batch == 0) return CONV_OK;
    const int es = dtype_size(desc->dtype);
    if (!x || !out || !aligned(x, es) || !aligned(out, es)) return CONV_EINVAL;
    if (x == out && (desc->ldx != desc->ldo || (desc->batch > 1 && desc->stride_x != desc->stride_o))) return CONV_EINVAL;
    OrthogonalArgs a = orthogonal_args(desc);
    if (!workspace || workspace_bytes < orthogonal_workspace(a, desc->dtype)) return CONV_EWORKSPACE;
    if (!aligned(workspace, 16)) return CONV_EINVAL;
    a.x = x, a.out = out, a.ws = workspace;
    return guarded("orthogonalize", [&] { return launch_orthogonalize(a, desc->dtype, (hipStream_t)stream); });
}

}  // extern "C"
