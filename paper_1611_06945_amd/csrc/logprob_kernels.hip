// Log probabilities of given tokens with entropy and the likeliest alternatives, and their gradient.
#include "rows_common.h"

namespace convfwd {

namespace {

constexpr float kInf = __builtin_inff();

// Whole numbers in the order of the floats: -0 equals +0, a NaN is above everything.
__device__ __forceinline__ uint32_t order_of(float x)
{
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
// ... and of (value, index): a lower index is greater.  Neither 0 nor all ones for an element, a NaN in column 0 included.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t j) { return ((uint64_t)order_of(x) << 32) | (0xFFFFFFFEu - j); }
__device__ __forceinline__ uint32_t index_of(uint64_t key) { return 0xFFFFFFFEu - (uint32_t)key; }

__device__ __forceinline__ uint64_t wave_max(uint64_t k)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const uint64_t o = __shfl_xor(k, d, 64);
        k = o > k ? o : k;
    }
    return k;
}

// A workgroup a row, the row read again for every pass and for every alternative: any length, any `top`.
template <int DT>
__global__ __launch_bounds__(256) void logprob_any(LogprobArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    __shared__ float red[3][4];
    __shared__ uint64_t best[2][4];
    const int tid = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    __syncthreads();
    const elem_t* x = (const elem_t*)a.x + row * a.ldx;
    float m = -kInf, bad = 0.0f;
    for (int j = tid; j < a.cols; j += 256) {
        const float v = Prec<DT>::to_f32(x[j]);
        m = fmaxf(m, v);
        if (!(v < kInf)) bad = 1.0f;
    }
    m = block_reduce<4, OpMax>(m, red[0]);
    bad = block_reduce<4, OpMax>(bad, red[1]);
    __syncthreads();
    const bool empty = m == -kInf && bad == 0.0f;
    float s = 0.0f, sd = 0.0f;
    for (int j = tid; j < a.cols; j += 256) {
        const float d = Prec<DT>::to_f32(x[j]) - m;
        const float e = expf(d);
        s += e;
        sd += e > 0.0f ? e * d : 0.0f;
    }
    s = block_reduce<4, OpSum>(s, red[0]);
    sd = block_reduce<4, OpSum>(sd, red[1]);
    float lse = m + logf(s), h = logf(s) - sd / s;
    if (empty) lse = -kInf, h = 0.0f;
    if (bad != 0.0f) lse = h = __builtin_nanf("");
    if (tid == 0) {
        if (a.lse) a.lse[row] = lse;
        if (a.entropy) a.entropy[row] = h;
        if (a.logp) {
            const int64_t t = a.target[row];
            a.logp[row] = t < 0 ? 0.0f : t >= a.cols ? __builtin_nanf("") : empty ? -kInf : Prec<DT>::to_f32(x[t]) - lse;
        }
    }
    uint64_t last = ~0ull;
    for (int i = 0; i < a.top; ++i) {
        uint64_t k = 0;
        for (int j = tid; j < a.cols; j += 256) {
            const uint64_t c = key_of(Prec<DT>::to_f32(x[j]), (uint32_t)j);
            if (c < last && c > k) k = c;
        }
        k = wave_max(k);
        if ((tid & 63) == 0) best[i & 1][tid >> 6] = k;
        __syncthreads();
        last = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) last = best[i & 1][w] > last ? best[i & 1][w] : last;
        if (tid == 0) {
            const uint32_t j = index_of(last);
            a.top_id[row * a.top + i] = (int64_t)j;
            a.top_logp[row * a.top + i] = empty ? -kInf : Prec<DT>::to_f32(x[j]) - lse;
        }
    }
    }
}

template <int DT>
__global__ __launch_bounds__(256) void logprob_bwd_any(LogprobArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const elem_t* x = (const elem_t*)a.x + row * a.ldx;
    elem_t* dx = (elem_t*)a.dx + row * a.ldg;
    const float lse = a.lse[row];
    const int64_t t = a.g_logp ? a.target[row] : -1;
    float g = t >= 0 ? a.g_logp[row] : 0.0f;
    if (t >= a.cols) g = __builtin_nanf("");
    const float gh = a.g_entropy ? a.g_entropy[row] : 0.0f, h = a.g_entropy ? a.entropy[row] : 0.0f;
    for (int j = threadIdx.x; j < a.cols; j += 256) {
        const float lp = Prec<DT>::to_f32(x[j]) - lse, p = expf(lp);
        float v = g * ((j == t ? 1.0f : 0.0f) - p);
        if (p > 0.0f) v -= gh * (p * (lp + h));
        dx[j] = Prec<DT>::from_f32(lse == -kInf ? 0.0f : v);
    }
    }
}

}  // namespace

size_t logprob_workspace(int64_t rows, int cols, int top) { return 0; }

hipError_t launch_logprob_fwd(LogprobArgs& a, int dtype, hipStream_t s)
{
    const dim3 grid((unsigned)(a.rows < (1 << 20) ? a.rows : 1 << 20)), block(256);
    if (dtype == CONV_F32) hipLaunchKernelGGL((logprob_any<CONV_F32>), grid, block, 0, s, a);
    else if (dtype == CONV_F16) hipLaunchKernelGGL((logprob_any<CONV_F16>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((logprob_any<CONV_BF16>), grid, block, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_logprob_bwd(LogprobArgs& a, int dtype, hipStream_t s)
{
    const dim3 grid((unsigned)(a.rows < (1 << 20) ? a.rows : 1 << 20)), block(256);
    if (dtype == CONV_F32) hipLaunchKernelGGL((logprob_bwd_any<CONV_F32>), grid, block, 0, s, a);
    else if (dtype == CONV_F16) hipLaunchKernelGGL((logprob_bwd_any<CONV_F16>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((logprob_bwd_any<CONV_BF16>), grid, block, 0, s, a);
    return hipGetLastError();
}

}  // namespace convfwd
