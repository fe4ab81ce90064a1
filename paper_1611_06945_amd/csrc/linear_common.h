// What the files of the linear layers share: the activations, what becomes of a sum, the launchers of products by operand type.
#pragma once

#include "product_kernel.h"

namespace convfwd {

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

// Phi(-|z|), Phi the normal distribution, and exp(-z^2 / 2).  It is exp(-z^2 / 2) t P(t) with t = 1 / (1 + c |z|), the form of formula 7.1.26 of Abramowitz and Stegun's
// handbook, with c and P fitted here for the least relative error; FINE up to |z| = 1 it is 1/2 - |z| Q(z^2).  (erff() takes four times the instructions.)  FINE is off by the roundings of
// fp32: GELU over normal z 3.1e-8 of the norm, with 1 + erf() in fp32 3.7e-8.  Otherwise by 1.1e-5 of the value at most, a fortieth of a rounding to fp16, for results that are stored
// in 16 bits; the handbook's own coefficients leave twice a rounding of fp16 at z = -3.5.  What a tile's 65536 activations cost is a part of its time (200704 x 192 x 768 fp16 with the
// sum kept 283 us, FINE 315), so divisions are reciprocals, off by a unit in the last place.
template <bool FINE>
__device__ __forceinline__ float normal_tail(float z, float& bell)
{
    const float u = fabsf(z), w = z * z;
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf((FINE ? 0.4f : 0.425f) * 0.70710678118654752f, u, 1.0f));
    bell = __builtin_amdgcn_exp2f(w * (-0.5f * 1.44269504088896341f));
    float p;
    if constexpr (!FINE) {
        p = __builtin_fmaf(-0.0769140348f, t, 0.213978097f);
        p = __builtin_fmaf(p, t, -0.014909937f);
        p = __builtin_fmaf(p, t, 0.143442242f);
        p = __builtin_fmaf(p, t, 0.114141129f);
        p = __builtin_fmaf(p, t, 0.120266527f);
        return p * t * bell;
    }
    p = __builtin_fmaf(-0.0566013232f, t, 0.117606282f);
    p = __builtin_fmaf(p, t, 0.00876443554f);
    p = __builtin_fmaf(p, t, 0.103900433f);
    p = __builtin_fmaf(p, t, 0.10019324f);
    p = __builtin_fmaf(p, t, 0.113221332f);
    p = __builtin_fmaf(p, t, 0.112821251f);
    float q = __builtin_fmaf(-7.65420828e-06f, w, 0.000113486371f);
    q = __builtin_fmaf(q, w, -0.00118632999f);
    q = __builtin_fmaf(q, w, 0.00997332297f);
    q = __builtin_fmaf(q, w, -0.0664903596f);
    q = __builtin_fmaf(q, w, 0.398942292f);
    return u < 1.0f ? __builtin_fmaf(-u, q, 0.5f) : p * t * bell;
}
// 1 / (1 + exp(-z))
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f)); }

// (Factors z beside a tail are clamped where the tail has vanished already: infinities give the limits, where they would give infinity times zero.)
// DT: what the value is stored as.
template <int DT>
__device__ __forceinline__ float act_of(float z, int act)
{
    if (act == ACT_RELU) return z < 0.0f ? 0.0f : z;  // a NaN stays
    if (act == ACT_GELU) {
        float bell;
        const float tail = normal_tail<DT == CONV_F32>(z, bell);
        return __builtin_fmaf(-fminf(fabsf(z), 16.0f), tail, z < 0.0f ? 0.0f : z);  // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
    }
    if (act == ACT_SILU) return fmaxf(z, -128.0f) * logistic(z);
    return z;
}
// its derivative, which goes into sums in fp32; 0 at the corner of ReLU
__device__ __forceinline__ float act_slope(float z, int act)
{
    if (act == ACT_RELU) return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
    if (act == ACT_GELU) {
        float bell;
        const float tail = normal_tail<true>(z, bell);
        return __builtin_fmaf(__builtin_amdgcn_fmed3f(z, -16.0f, 16.0f) * bell, 0.39894228040143268f, z < 0.0f ? tail : 1.0f - tail);
    }
    if (act == ACT_SILU) {
        const float p = logistic(z);
        return p * __builtin_fmaf(__builtin_amdgcn_fmed3f(z, -128.0f, 128.0f), 1.0f - p, 1.0f);
    }
    return 1.0f;
}

// out = act(sum + bias) + residual, and the sum with its bias where it is asked for.
struct LinearOut {
    const float* bias;
    const void* residual;
    void* pre;
    void* out;
    int64_t ldr, ldo;
    int act;
};

template <int DT>
struct LinearEpi {
    typedef LinearOut Args;
    static constexpr bool SYMMETRIC = false;
    static __device__ __forceinline__ void prepare(const Args& e, float* bias, int64_t n0, int here, int width, int threads)
    {
        for (int i = threadIdx.x; i < width; i += threads) bias[i] = e.bias && i < here ? e.bias[n0 + i] : 0.0f;
    }
    template <int W>
    static __device__ __forceinline__ void finish(const ProductArgs&, const Args& e, float (&v)[W], int64_t m, int64_t n, int have, const float* bias)
    {
        if (e.bias) {
#pragma unroll
            for (int k = 0; k < W; ++k) v[k] += bias[k];
        }
        if (e.pre) put_pieces<DT, W>(e.pre, m * e.ldo + n, v, have);
        if (e.act) {
#pragma unroll
            for (int k = 0; k < W; ++k) v[k] = act_of<DT>(v[k], e.act);
        }
        if (e.residual) {
            float r[W];
            get_pieces<DT, W>(e.residual, m * e.ldr + n, r, have);
#pragma unroll
            for (int k = 0; k < W; ++k) v[k] += r[k];
        }
        put_pieces<DT, W>(e.out, m * e.ldo + n, v, have);
    }
};

// Tiles of a product; the last two are for operands that start anywhere.
enum ProductForm { P64, P128, P256, P192, P64_ANY, P128_ANY };
typedef ProductTile<4, 2, 1, 2, 4> Tile64;
typedef ProductTile<2, 4, 4, 2, 2> Tile128;  // two workgroups a CU
typedef ProductTile<4, 2, 4, 8, 2> Tile256;
typedef ProductTile<4, 2, 3, 6, 3> Tile192;
typedef ProductTile<4, 2, 1, 2, 2> Tile64Any;

enum ProductLayout { LAYOUT_NT, LAYOUT_NN, LAYOUT_TN };  // which operand lies across the reduction: none, the second, both

// The products of fp16, bf16 and fp32 rows (fp32: strides in elements of four bytes, tiles of 64 x 64, 128 x 128 and 256 x 128).  splits > 1: partial sums to g.partial.
hipError_t launch_product_f16(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s);
hipError_t launch_product_bf16(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s);
hipError_t launch_product_f32(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s);
// ... of a first operand in two parts (LAYOUT_NN and LAYOUT_TN: the gradients behind GELU and SiLU).
hipError_t launch_product_parts_f16(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s);
hipError_t launch_product_parts_bf16(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s);

template <int DT, typename T, bool A_ACROSS, bool B_ACROSS, bool DIRECT, typename Epi, bool PARTS = false>
hipError_t launch_product_tiles(ProductArgs g, const typename Epi::Args& e, int batch, int splits, hipStream_t s)
{
    const void* f = (const void*)product_kernel<DT, T, A_ACROSS, B_ACROSS, DIRECT, Epi, PARTS>;
    const hipError_t err = ensure_dynamic_lds(f, T::LDS);
    if (err != hipSuccess) return err;
    g.tiles_n = (int)((g.N + T::BN - 1) / T::BN);
    g.each = (g.ksteps + splits - 1) / splits, g.splits = splits;
    // a launch holds less than 2^32 threads: the rows go in portions of so many tiles (the triangle of a symmetric product, of a side up to 2^17, in one)
    const int64_t all = g.M, bands = Epi::SYMMETRIC ? g.tiles_n : std::max<int64_t>(1, (1 << 21) / ((int64_t)g.tiles_n * batch * splits));
    for (int64_t skip = 0; skip < all; skip += bands * T::BT) {
        ProductArgs p = g;
        p.M = std::min(bands * T::BT, all - skip), p.m_first = skip;
        p.a += A_ACROSS ? skip : skip * g.lda;
        p.tiles_m = (int)((p.M + T::BT - 1) / T::BT);
        const unsigned tiles = Epi::SYMMETRIC ? (unsigned)((int64_t)p.tiles_m * (p.tiles_m + 1) / 2) : (unsigned)p.tiles_m * (unsigned)p.tiles_n;
        hipLaunchKernelGGL((product_kernel<DT, T, A_ACROSS, B_ACROSS, DIRECT, Epi, PARTS>), dim3(tiles * (unsigned)splits, (unsigned)batch), dim3(T::NT), T::LDS, s, p, e);
    }
    return hipGetLastError();
}

template <int DT, bool A_ACROSS, bool B_ACROSS, typename Epi, bool PARTS = false>
hipError_t launch_product_form(const ProductArgs& g, const typename Epi::Args& e, ProductForm form, int batch, int splits, hipStream_t s)
{
    switch (form) {
        case P64: return launch_product_tiles<DT, Tile64, A_ACROSS, B_ACROSS, true, Epi, PARTS>(g, e, batch, splits, s);
        case P128: return launch_product_tiles<DT, Tile128, A_ACROSS, B_ACROSS, true, Epi, PARTS>(g, e, batch, splits, s);
        case P256: return launch_product_tiles<DT, Tile256, A_ACROSS, B_ACROSS, true, Epi, PARTS>(g, e, batch, splits, s);
        case P192: return launch_product_tiles<DT, Tile192, A_ACROSS, B_ACROSS, true, Epi, PARTS>(g, e, batch, splits, s);
        case P64_ANY: return launch_product_tiles<DT, Tile64Any, A_ACROSS, B_ACROSS, false, Epi, PARTS>(g, e, batch, splits, s);
        default: return launch_product_tiles<DT, Tile128, A_ACROSS, B_ACROSS, false, Epi, PARTS>(g, e, batch, splits, s);
    }
}

#define CONVFWD_PRODUCT_LAYOUTS(launch, DT, Epi)                                                   \
    switch (layout) {                                                                              \
        case LAYOUT_NT: return launch<DT, false, false, Epi>(g, arg, form, 1, splits, s);          \
        case LAYOUT_NN: return launch<DT, false, true, Epi>(g, arg, form, 1, splits, s);           \
        default: return launch<DT, true, true, Epi>(g, arg, form, 1, splits, s);                   \
    }

#define CONVFWD_PARTS_LAYOUTS(launch, DT, Epi)                                                       \
    return layout == LAYOUT_NN ? launch<DT, false, true, Epi, true>(g, arg, form, 1, splits, s)      \
                               : launch<DT, true, true, Epi, true>(g, arg, form, 1, splits, s);

}  // namespace convfwd
