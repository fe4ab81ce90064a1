// Layer norm forward and backward, and the row quantiser.
#include <algorithm>

#include "rows_common.h"

namespace convfwd {

namespace {

constexpr float kInv127 = 1.0f / 127.0f;
constexpr float kLeastScale = 0x1p-126f;

// The scale of a row with the largest magnitude `amax` (NaN or inf where the row holds one), and what its elements are
// multiplied with.  The scale is kept from the denormal numbers, so its reciprocal is finite.
struct RowScale {
    float scale, inv;
    bool good;
};
__device__ __forceinline__ RowScale row_scale(float amax)
{
    RowScale r;
    r.good = amax < __builtin_inff();
    r.scale = fmaxf(amax * kInv127, kLeastScale);
    r.inv = 1.0f / r.scale;
    if (!r.good) r.scale = __builtin_nanf(""), r.inv = 0.0f;
    return r;
}
__device__ __forceinline__ int code(float x, const RowScale& r) { return r.good ? (int)__builtin_rintf(x * r.inv) : 0; }
// magnitude for a maximum that must not lose a NaN: ordered by its bits, where NaN is above infinity
__device__ __forceinline__ float keep(float m, float x)
{
    const uint32_t a = __builtin_bit_cast(uint32_t, m), b = __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu;
    return __builtin_bit_cast(float, a > b ? a : b);
}
struct OpKeep {
    static __device__ __forceinline__ float of(float a, float b) { return keep(a, b); }
};

// A workgroup a row, the row read again for every pass: rows of any length.
template <int DT>
__global__ __launch_bounds__(256) void norm_fwd_any(NormArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    __shared__ float red[3][4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    __syncthreads();
    const elem_t* x = (const elem_t*)a.x + row * a.ldx;
    float sum = 0.0f;
    for (int j = threadIdx.x; j < a.cols; j += 256) sum += Prec<DT>::to_f32(x[j]);
    const float mean = block_reduce<4, OpSum>(sum, red[0]) / (float)a.cols;
    float sq = 0.0f;
    for (int j = threadIdx.x; j < a.cols; j += 256) {
        const float d = Prec<DT>::to_f32(x[j]) - mean;
        sq = __builtin_fmaf(d, d, sq);
    }
    const float rstd = 1.0f / sqrtf(block_reduce<4, OpSum>(sq, red[1]) / (float)a.cols + a.eps);
    auto value = [&](int j) {
        float v = (Prec<DT>::to_f32(x[j]) - mean) * rstd;
        if (a.gamma) v *= a.gamma[j];
        if (a.beta) v += a.beta[j];
        return Prec<DT>::from_f32(v);
    };
    if (!a.q) {
        elem_t* y = (elem_t*)a.y + row * a.ldy;
        for (int j = threadIdx.x; j < a.cols; j += 256) y[j] = value(j);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        continue;
    }
    float amax = 0.0f;
    for (int j = threadIdx.x; j < a.cols; j += 256) amax = keep(amax, Prec<DT>::to_f32(value(j)));
    const RowScale r = row_scale(block_reduce<4, OpKeep>(amax, red[2]));
    int8_t* q = a.q + row * a.ldy;
    const int padded = (a.cols + 15) & ~15;
    for (int j = threadIdx.x; j < padded; j += 256) q[j] = j < a.cols ? (int8_t)code(Prec<DT>::to_f32(value(j)), r) : (int8_t)0;
    if (threadIdx.x == 0) a.scale[row] = r.scale;
    }
}

template <int DT>
__global__ __launch_bounds__(256) void quant_any(QuantArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    __shared__ float red[4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    __syncthreads();
    const elem_t* x = (const elem_t*)a.x + row * a.ldx;
    float amax = 0.0f;
    for (int j = threadIdx.x; j < a.cols; j += 256) amax = keep(amax, Prec<DT>::to_f32(x[j]));
    const RowScale r = row_scale(block_reduce<4, OpKeep>(amax, red));
    int8_t* q = a.q + row * a.ldq;
    const int padded = (a.cols + 15) & ~15;
    for (int j = threadIdx.x; j < padded; j += 256) q[j] = j < a.cols ? (int8_t)code(Prec<DT>::to_f32(x[j]), r) : (int8_t)0;
    if (threadIdx.x == 0) a.scale[row] = r.scale;
    }
}

template <int DT>
__global__ __launch_bounds__(256) void norm_dx_any(NormArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    __shared__ float red[2][4];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    __syncthreads();
    const elem_t* x = (const elem_t*)a.x + row * a.ldx;
    const elem_t* dy = (const elem_t*)a.dy + row * a.ldy;
    elem_t* dx = (elem_t*)a.dx + row * a.ldx;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int j = threadIdx.x; j < a.cols; j += 256) {
        const float g = Prec<DT>::to_f32(dy[j]) * (a.gamma ? a.gamma[j] : 1.0f);
        s1 += g;
        s2 = __builtin_fmaf(g, (Prec<DT>::to_f32(x[j]) - mean) * rstd, s2);
    }
    const float c1 = block_reduce<4, OpSum>(s1, red[0]) / (float)a.cols;
    const float c2 = block_reduce<4, OpSum>(s2, red[1]) / (float)a.cols;
    for (int j = threadIdx.x; j < a.cols; j += 256) {
        const float g = Prec<DT>::to_f32(dy[j]) * (a.gamma ? a.gamma[j] : 1.0f);
        const float xh = (Prec<DT>::to_f32(x[j]) - mean) * rstd;
        dx[j] = Prec<DT>::from_f32(rstd * (g - c1 - xh * c2));
    }
    }
}

// dgamma and dbeta: a thread a column, gridDim.y workgroups share the rows.
template <int DT>
__global__ __launch_bounds__(256) void norm_dw_any(NormArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= a.cols) return;
    float dg = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float g = Prec<DT>::to_f32(((const elem_t*)a.dy)[row * a.ldy + j]);
        dg = __builtin_fmaf(g, (Prec<DT>::to_f32(((const elem_t*)a.x)[row * a.ldx + j]) - a.mean[row]) * a.rstd[row], dg);
        db += g;
    }
    a.ws[((size_t)blockIdx.y * 2) * a.cols + j] = dg;
    a.ws[((size_t)blockIdx.y * 2 + 1) * a.cols + j] = db;
}

// The partial sums of `parts` workgroups, in order.
__global__ __launch_bounds__(256) void norm_dw_join(NormArgs a, int parts)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= a.cols) return;
    float dg = 0.0f, db = 0.0f;
    for (int p = 0; p < parts; ++p) {
        dg += a.ws[((size_t)p * 2) * a.cols + j];
        db += a.ws[((size_t)p * 2 + 1) * a.cols + j];
    }
    if (a.dgamma) a.dgamma[j] = dg;
    if (a.dbeta) a.dbeta[j] = db;
}

// one workgroup a row up to 2^20 of them, which then take several
unsigned row_grid(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 1 << 20); }

int dw_parts(int64_t rows) { return (int)std::min<int64_t>(64, (rows + 15) / 16); }

template <int DT>
hipError_t bwd(NormArgs& a, hipStream_t s)
{
    if (a.dgamma || a.dbeta) {
        const int parts = dw_parts(a.rows);
        const unsigned cb = (unsigned)((a.cols + 255) / 256);
        if (parts) hipLaunchKernelGGL((norm_dw_any<DT>), dim3(cb, parts), dim3(256), 0, s, a);
        hipLaunchKernelGGL(norm_dw_join, dim3(cb), dim3(256), 0, s, a, parts);
    }
    if (a.dx && a.rows) hipLaunchKernelGGL((norm_dx_any<DT>), dim3(row_grid(a.rows)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

size_t layernorm_bwd_workspace(int64_t rows, int cols, int dtype) { return (size_t)dw_parts(rows) * 2 * cols * 4; }

hipError_t launch_layernorm_fwd(NormArgs& a, int dtype, hipStream_t s)
{
    const dim3 grid(row_grid(a.rows)), block(256);
    if (dtype == CONV_F32) hipLaunchKernelGGL((norm_fwd_any<CONV_F32>), grid, block, 0, s, a);
    else if (dtype == CONV_F16) hipLaunchKernelGGL((norm_fwd_any<CONV_F16>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((norm_fwd_any<CONV_BF16>), grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_quantize_rows(QuantArgs& a, int dtype, hipStream_t s)
{
    const dim3 grid(row_grid(a.rows)), block(256);
    if (dtype == CONV_F32) hipLaunchKernelGGL((quant_any<CONV_F32>), grid, block, 0, s, a);
    else if (dtype == CONV_F16) hipLaunchKernelGGL((quant_any<CONV_F16>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((quant_any<CONV_BF16>), grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_layernorm_bwd(NormArgs& a, int dtype, hipStream_t s)
{
    return dtype == CONV_F32 ? bwd<CONV_F32>(a, s) : dtype == CONV_F16 ? bwd<CONV_F16>(a, s) : bwd<CONV_BF16>(a, s);
}

}  // namespace convfwd
