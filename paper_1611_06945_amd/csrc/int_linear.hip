// Matrix product in 8-bit integers with scales for each row and output channel.
#include "rows_common.h"

namespace convfwd {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// The first `n` bytes of a 16-byte piece (n may be <= 0 or >= 16), the others zero.
__device__ __forceinline__ uint4 first_bytes(uint4 v, int n)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int have = n - 4 * i;
        w[i] = have >= 4 ? w[i] : have <= 0 ? 0u : w[i] & ((1u << (8 * have)) - 1u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int DT>
__device__ __forceinline__ typename Prec<DT>::elem_t finish(int acc, float scale, float bias, int relu)
{
    float v = (float)acc * scale + bias;
    if (relu) v = v < 0.0f ? 0.0f : v;  // a NaN stays
    return Prec<DT>::from_f32(v);
}

// A wave 16 channels x 16 rows, operands from memory straight into registers.
template <int DT>
__global__ __launch_bounds__(256) void int_linear_tile16(IntLinearArgs g)
{
    typedef typename Prec<DT>::elem_t elem_t;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = (blockIdx.x * 4 + wave) * 16;
    const int64_t t0 = (int64_t)blockIdx.y * 16;
    if (n0 >= g.N) return;
    const int i = lane & 15, kq = (lane >> 4) * 16;
    const int8_t* w = g.w + (int64_t)min(n0 + i, g.N - 1) * g.ldw;
    const int8_t* a = g.a + (t0 + i < g.rows ? t0 + i : g.rows - 1) * g.lda;
    i32x4 acc = {0, 0, 0, 0};
    for (int k = kq; k - kq < g.K; k += 64) {
        uint4 wv = make_uint4(0, 0, 0, 0), av = wv;
        if (k < g.K) {
            wv = first_bytes(*(const uint4*)(w + k), g.K - k);
            av = *(const uint4*)(a + k);
        }
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, wv), __builtin_bit_cast(i32x4, av), acc, 0, 0, 0);
    }
    const int64_t t = t0 + i;
    if (t >= g.rows) return;
    const float sa = g.a_scale[t];
    elem_t* out = (elem_t*)g.out + t * g.ldo;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int n = n0 + (lane >> 4) * 4 + r;
        if (n < g.N) out[n] = finish<DT>(acc[r], sa * g.w_scale[n], g.bias ? g.bias[n] : 0.0f, g.relu);
    }
}

}  // namespace

size_t int_linear_workspace(int64_t rows, int N, int K) { return 0; }

hipError_t launch_int_linear(IntLinearArgs& g, int dtype, hipStream_t s)
{
    const int64_t nt = (g.rows + 15) / 16;
    const dim3 block(256);
    // gridDim.y is at most 65535: the rows go in portions
    for (int64_t t = 0; t < nt; t += 65535) {
        IntLinearArgs p = g;
        const int64_t skip = t * 16, left = g.rows - skip;
        p.rows = left < 65535 * 16 ? left : 65535 * 16;
        p.a += skip * g.lda, p.a_scale += skip, p.out = (char*)g.out + skip * g.ldo * dtype_size(dtype);
        const dim3 grid((unsigned)((g.N + 63) / 64), (unsigned)((p.rows + 15) / 16));
        if (dtype == CONV_F32) hipLaunchKernelGGL((int_linear_tile16<CONV_F32>), grid, block, 0, s, p);
        else if (dtype == CONV_F16) hipLaunchKernelGGL((int_linear_tile16<CONV_F16>), grid, block, 0, s, p);
        else hipLaunchKernelGGL((int_linear_tile16<CONV_BF16>), grid, block, 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace convfwd
