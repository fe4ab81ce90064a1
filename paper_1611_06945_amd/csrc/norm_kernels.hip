// Layer norm forward and backward, and the row quantiser: one pass over the tensors, the row held in registers.
//
// G neighbouring lanes share a row (8, 16, a wave, or several: forward a workgroup of as many as the row takes, G = 0, backward 4 or 8),
// each holding up to NV pieces of 16 bytes.  The mean comes first and the variance is summed around it, from registers.  A workgroup keeps
// its columns' gamma and beta in registers over all its rows, and asks for its next row before it works on the present one.  Backward, a lane adds up dgamma and dbeta of its columns
// over its rows in registers; a workgroup's lanes with the same columns are added through LDS, and a second kernel adds the
// workgroups' sums, always in the same order.  Longer rows are read again for every pass (`_any`): forward from 32768 columns of
// 16 bits and 16384 of fp32 on (32 and 16 elements a lane of 16 waves), backward from 16384 (32 of 8 waves).
#include <algorithm>

#include "held_rows.h"

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

// The largest magnitude among stored values, as `keep` has it.  In 16 bits two at a time: without the sign the bits of numbers, inf
// and NaN are in order.
template <int DT, int NV>
__device__ __forceinline__ float largest(const uint4 (&raw)[NV])
{
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    const uint32_t clear = DT == CONV_F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (DT == CONV_F32) m = max(m, w[k] & clear);
            else m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, m), __builtin_bit_cast(us2, w[k] & clear)));
        }
    }
    if constexpr (DT == CONV_F32) return __builtin_bit_cast(float, m);
    else return Prec<DT>::to_f32((typename Prec<DT>::elem_t)max(m & 0xFFFFu, m >> 16));
}

// Codes of a piece to q.  Pieces past the end up to the next multiple of 16 columns get zeros.  The codes are rint(v * inv): added to
// 1.5 * 2^23, the product is rounded to the integers and its low byte is the code.
template <int VEC>
__device__ __forceinline__ void store_codes(int8_t* q, const float (&v)[VEC], const RowScale& r, int j, int padded)
{
#pragma clang fp contract(off)
    if (j >= padded) return;
    uint32_t w[VEC / 4];
#pragma unroll
    for (int k = 0; k < VEC / 4; ++k) {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p = v[k * 4 + e] * r.inv;
            u[e] = __builtin_bit_cast(uint32_t, p + 0x1.8p23f);
        }
        const uint32_t all = __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0C0C0400), __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0400), 0x05040100);
        w[k] = r.good ? all : 0;
    }
    __builtin_memcpy(__builtin_assume_aligned(q + j, VEC), w, VEC);
}

enum { TO_FLOAT = 0, TO_CODES = 1, QUANT_ONLY = 2 };

// Layer norm (to floats or codes), or the quantiser alone, which holds rows the same way.
template <int DT, int G, int NV, int MODE>
__global__ __launch_bounds__(G ? 256 : 1024) void norm_fwd_rows(NormArgs a)
{
    typedef Held<DT, G, NV> H;
    typedef typename H::elem_t elem_t;
    constexpr int VEC = H::VEC, ROWS = G ? 256 / G : 1;
    __shared__ float red[3][G ? 1 : 16];
    const int l = G ? threadIdx.x % G : threadIdx.x;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + (G ? threadIdx.x / G : 0);
    const int padded = (a.cols + 15) & ~15;
    const float inv_cols = 1.0f / (float)a.cols;
    auto load = [&](uint4 (&raw)[NV], int64_t r) { H::load(raw, (const elem_t*)a.x + (r < a.rows ? r : a.rows - 1) * a.ldx, a.cols, l); };

    constexpr bool AHEAD = NV * VEC < 32;  // (no registers for the next row: 16 waves with 32 elements a lane)
    uint4 next[NV];
    if (AHEAD) load(next, row);
    float gamma[NV][VEC], beta[NV][VEC];
    if constexpr (MODE != QUANT_ONLY) {
        H::columns(gamma, a.gamma, 1.0f, a.cols, l);
        H::columns(beta, a.beta, 0.0f, a.cols, l);
    }
    // every lane of a workgroup makes the same number of rounds: the reductions of wide rows have barriers
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += step, row += step) {
        if (!AHEAD) load(next, row);
        float x[NV][VEC];
        uint4 raw[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i] = next[i];
        H::clear(raw, a.cols, l);
        if (AHEAD && first + step < a.rows) load(next, row + step);
#pragma unroll
        for (int i = 0; i < NV; ++i) H::P::widen(raw[i], x[i]);
        if constexpr (MODE != QUANT_ONLY) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) sum += x[i][k];
            const float mean = row_reduce<G, OpSum>(sum, red[0]) * inv_cols;
            float sq = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int left = a.cols - (i * H::lanes() + l) * VEC;
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    x[i][k] -= mean;
                    if (left < VEC) x[i][k] = k < left ? x[i][k] : 0.0f;
                    sq = __builtin_fmaf(x[i][k], x[i][k], sq);
                }
            }
            const float rstd = 1.0f / sqrtf(row_reduce<G, OpSum>(sq, red[1]) * inv_cols + a.eps);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) x[i][k] = __builtin_fmaf(x[i][k] * rstd, gamma[i][k], beta[i][k]);
            if constexpr (MODE == TO_FLOAT) {
                if (row < a.rows) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) H::store((elem_t*)a.y + row * a.ldy, x[i], a.cols, i, l);
                    if (l == 0) {
                        if (a.mean) a.mean[row] = mean;
                        if (a.rstd) a.rstd[row] = rstd;
                    }
                }
            } else {
                // the codes are those of the rounded values
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    raw[i] = H::P::narrow(x[i]);
                    H::P::widen(raw[i], x[i]);
                }
            }
        }
        if constexpr (MODE != TO_FLOAT) {
            // (past the end gamma is 1 and beta 0, so zeros have stayed zeros)
            const RowScale r = row_scale(row_reduce<G, OpKeep>(largest<DT>(raw), red[2]));
            if (row < a.rows) {
#pragma unroll
                for (int i = 0; i < NV; ++i) store_codes<VEC>(a.q + row * a.ldy, x[i], r, (i * H::lanes() + l) * VEC, padded);
                if (l == 0) a.scale[row] = r.scale;
            }
        }
        if constexpr (G == 0) __syncthreads();  // the next row's reductions use the same LDS
    }
}

// Backward.  DX: dx is asked for; DW: dgamma or dbeta is.  A workgroup's sums go to ws, or, where there is one workgroup only, to their place.
template <int DT, int G, int NV, int NT, bool DX, bool DW>
__global__ __launch_bounds__(NT) void norm_bwd_rows(NormArgs a)
{
    typedef Held<DT, G, NV> H;
    typedef typename H::elem_t elem_t;
    constexpr int VEC = H::VEC, ROWS = NT / G, WAVES = NT / 64, SETS = G <= 64 ? WAVES : ROWS;
    __shared__ float red[2][WAVES];
    __shared__ float sums[DW && SETS > 1 ? SETS / 2 * 2 * G * NV * VEC : 1];
    const int tid = threadIdx.x, l = tid % G;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + tid / G;
    const float inv_cols = 1.0f / (float)a.cols;
    auto clamp = [&](int64_t r) { return r < a.rows ? r : a.rows - 1; };

    uint4 nx[NV], ndy[NV];
    float nmean, nrstd;
    auto fetch = [&](int64_t r) {
        r = clamp(r);
        H::load(nx, (const elem_t*)a.x + r * a.ldx, a.cols, l);
        H::load(ndy, (const elem_t*)a.dy + r * a.ldy, a.cols, l);
        nmean = a.mean[r], nrstd = a.rstd[r];
    };
    constexpr bool AHEAD = NV * VEC < 32;
    if (AHEAD && a.rows) fetch(row);
    float gamma[NV][VEC], dg[NV][VEC], db[NV][VEC];
    if constexpr (DX) H::columns(gamma, a.gamma, 1.0f, a.cols, l);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int k = 0; k < VEC; ++k) dg[i][k] = db[i][k] = 0.0f;

    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += step, row += step) {
        if (!AHEAD) fetch(row);
        float x[NV][VEC], dy[NV][VEC];
        const float mean = nmean, rstd = nrstd;
        H::clear(nx, a.cols, l);
        H::clear(ndy, a.cols, l);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            H::P::widen(nx[i], x[i]);
            H::P::widen(ndy[i], dy[i]);
        }
        if (AHEAD && first + step < a.rows) fetch(row + step);
        const bool in = row < a.rows;
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                x[i][k] = (x[i][k] - mean) * rstd;  // past the end dy is 0
                if constexpr (DW) {
                    if (in) {
                        dg[i][k] = __builtin_fmaf(dy[i][k], x[i][k], dg[i][k]);
                        db[i][k] += dy[i][k];
                    }
                }
                if constexpr (DX) {
                    dy[i][k] *= gamma[i][k];
                    s1 += dy[i][k];
                    s2 = __builtin_fmaf(dy[i][k], x[i][k], s2);
                }
            }
        if constexpr (DX) {
            float c1, c2;
            if constexpr (G <= 64) {
                c1 = lanes_reduce<G, OpSum>(s1) * inv_cols, c2 = lanes_reduce<G, OpSum>(s2) * inv_cols;
            } else {
                // the waves of this row; other rows of the workgroup have waves of their own
                constexpr int W = G / 64;
                s1 = lanes_reduce<64, OpSum>(s1), s2 = lanes_reduce<64, OpSum>(s2);
                const int wave = tid >> 6, w0 = wave / W * W;
                if ((tid & 63) == 0) red[0][wave] = s1, red[1][wave] = s2;
                __syncthreads();
                s1 = red[0][w0], s2 = red[1][w0];
#pragma unroll
                for (int w = 1; w < W; ++w) s1 += red[0][w0 + w], s2 += red[1][w0 + w];
                c1 = s1 * inv_cols, c2 = s2 * inv_cols;
                __syncthreads();
            }
            if (in) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float v[VEC];
#pragma unroll
                    for (int k = 0; k < VEC; ++k) v[k] = rstd * (dy[i][k] - c1 - x[i][k] * c2);
                    H::store((elem_t*)a.dx + row * a.ldx, v, a.cols, i, l);
                }
            }
        }
    }
    if constexpr (DW) {
        // rows within a wave first, then halves of the waves (or rows) hand theirs to the others through LDS
        if constexpr (G < 64) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    dg[i][k] = across_rows<G>(dg[i][k]);
                    db[i][k] = across_rows<G>(db[i][k]);
                }
        }
        const int set = G <= 64 ? tid / 64 : tid / G;
        const bool holder = G >= 64 || (tid & 63) < G;
#pragma unroll
        for (int half = SETS / 2; half >= 1; half /= 2) {
            float* p = sums + (set % half) * (2 * G * NV * VEC) + l;  // a lane's neighbours are next to it: no bank twice
            if (set >= half && set < 2 * half && holder) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        p[(i * VEC + k) * G] = dg[i][k];
                        p[((NV + i) * VEC + k) * G] = db[i][k];
                    }
            }
            __syncthreads();
            if (set < half && holder) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        dg[i][k] += p[(i * VEC + k) * G];
                        db[i][k] += p[((NV + i) * VEC + k) * G];
                    }
            }
            if (half > 1) __syncthreads();
        }
        if (set == 0 && holder) {
            float* to_dg = gridDim.x == 1 ? a.dgamma : a.ws + (size_t)blockIdx.x * 2 * a.cols;
            float* to_db = gridDim.x == 1 ? a.dbeta : a.ws + (size_t)blockIdx.x * 2 * a.cols + a.cols;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = (i * H::lanes() + l) * VEC;
                if (j + VEC <= a.cols) {
                    if (to_dg) __builtin_memcpy(to_dg + j, dg[i], 4 * VEC);
                    if (to_db) __builtin_memcpy(to_db + j, db[i], 4 * VEC);
                } else {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        if (j + k < a.cols && to_dg) to_dg[j + k] = dg[i][k];
                        if (j + k < a.cols && to_db) to_db[j + k] = db[i][k];
                    }
                }
            }
        }
    }
}

// The sums of `parts` workgroups: C columns and 1024 / C groups of lanes a workgroup, a group every so many parts, then the groups in order.
template <int C>
__global__ __launch_bounds__(1024) void norm_dw_join(NormArgs a, int parts, int64_t from)
{
    constexpr int GROUPS = 1024 / C;
    __shared__ float red[GROUPS][C];
    const int l = threadIdx.x % C, group = threadIdx.x / C;
    const int64_t j = from + (int64_t)blockIdx.x * C + l;  // dgamma's columns, then dbeta's
    float s = 0.0f;
    if (j < 2 * (int64_t)a.cols) {
        int p = group;
        for (; p + 3 * GROUPS < parts; p += 4 * GROUPS) {
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = a.ws[(size_t)(p + GROUPS * u) * 2 * a.cols + j];
#pragma unroll
            for (int u = 0; u < 4; ++u) s += v[u];
        }
        for (; p < parts; p += GROUPS) s += a.ws[(size_t)p * 2 * a.cols + j];
    }
    red[group][l] = s;
    __syncthreads();
    if (group == 0 && j < 2 * (int64_t)a.cols) {
        float v[16];
#pragma unroll
        for (int g = 0; g < GROUPS; g += 16) {
#pragma unroll
            for (int u = 0; u < 16; ++u) v[u] = red[g + u][l];
#pragma unroll
            for (int u = 0; u < 16; ++u) s = g + u ? s + v[u] : v[u];
        }
        float* to = j < a.cols ? a.dgamma : a.dbeta;
        if (to) to[j < a.cols ? j : j - a.cols] = s;
    }
}

// ---- rows of any length: a workgroup a row, the row read again for every pass --------------------------------------------
// An element a load, three passes forward and two backward (and one more for the columns' sums), most of them from cache: 1310 x 20000 fp32
// forward 67 us (3.1 TB/s of what has to be read and written), to 8 bits 85, backward 122; 1310 x 40000 bf16 115, 158 and 171.

template <int DT, int MODE>
__global__ __launch_bounds__(1024) void norm_fwd_any(NormArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    constexpr int NT = 1024;
    __shared__ float red[3][16];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const elem_t* x = (const elem_t*)a.x + row * a.ldx;
        float mean = 0.0f, rstd = 1.0f;
        if constexpr (MODE != QUANT_ONLY) {
            float sum = 0.0f, sq = 0.0f;
            for (int j = threadIdx.x; j < a.cols; j += NT) sum += Prec<DT>::to_f32(x[j]);
            mean = block_reduce<16, OpSum>(sum, red[0]) / (float)a.cols;
            for (int j = threadIdx.x; j < a.cols; j += NT) {
                const float d = Prec<DT>::to_f32(x[j]) - mean;
                sq = __builtin_fmaf(d, d, sq);
            }
            rstd = 1.0f / sqrtf(block_reduce<16, OpSum>(sq, red[1]) / (float)a.cols + a.eps);
        }
        auto value = [&](int j) -> elem_t {
            if constexpr (MODE == QUANT_ONLY) return x[j];
            return Prec<DT>::from_f32(__builtin_fmaf((Prec<DT>::to_f32(x[j]) - mean) * rstd, a.gamma ? a.gamma[j] : 1.0f, a.beta ? a.beta[j] : 0.0f));
        };
        if constexpr (MODE == TO_FLOAT) {
            elem_t* y = (elem_t*)a.y + row * a.ldy;
            for (int j = threadIdx.x; j < a.cols; j += NT) y[j] = value(j);
            if (threadIdx.x == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        } else {
            float amax = 0.0f;
            for (int j = threadIdx.x; j < a.cols; j += NT) amax = keep(amax, Prec<DT>::to_f32(value(j)));
            const RowScale r = row_scale(block_reduce<16, OpKeep>(amax, red[2]));
            int8_t* q = a.q + row * a.ldy;
            const int padded = (a.cols + 15) & ~15;
            for (int j = threadIdx.x; j < padded; j += NT) q[j] = j < a.cols ? (int8_t)code(Prec<DT>::to_f32(value(j)), r) : (int8_t)0;
            if (threadIdx.x == 0) a.scale[row] = r.scale;
        }
        __syncthreads();
    }
}

template <int DT>
__global__ __launch_bounds__(1024) void norm_dx_any(NormArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    constexpr int NT = 1024;
    __shared__ float red[2][16];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const elem_t* x = (const elem_t*)a.x + row * a.ldx;
        const elem_t* dy = (const elem_t*)a.dy + row * a.ldy;
        elem_t* dx = (elem_t*)a.dx + row * a.ldx;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int j = threadIdx.x; j < a.cols; j += NT) {
            const float g = Prec<DT>::to_f32(dy[j]) * (a.gamma ? a.gamma[j] : 1.0f);
            s1 += g;
            s2 = __builtin_fmaf(g, (Prec<DT>::to_f32(x[j]) - mean) * rstd, s2);
        }
        const float c1 = block_reduce<16, OpSum>(s1, red[0]) / (float)a.cols;
        const float c2 = block_reduce<16, OpSum>(s2, red[1]) / (float)a.cols;
        for (int j = threadIdx.x; j < a.cols; j += NT) {
            const float g = Prec<DT>::to_f32(dy[j]) * (a.gamma ? a.gamma[j] : 1.0f);
            const float xh = (Prec<DT>::to_f32(x[j]) - mean) * rstd;
            dx[j] = Prec<DT>::from_f32(rstd * (g - c1 - xh * c2));
        }
        __syncthreads();
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

// ---- which form -------------------------------------------------------------------------------------------------------

constexpr int kCUs = 256;

// Backward: the fewest lanes that hold the row with 16 elements each; a wave and more of 16-bit rows 24, so that fewer are idle (us with 16 / 24:
// 43690 x 1152 bf16 77 / 61, 2000 x 1536 bf16 14 / 12; fp32, whose next row takes twice the registers, 32768 x 1536 108 / 124).  The longest
// have 512 lanes with up to 32, the 32 without the next row (which spilled 90 registers): 5225 x 9632 bf16 65 us, 4096 x 12288
// 67, where 16 waves with 16 a lane took 87 and 77.  lanes 0: the row is too long.
struct Form {
    int lanes, pieces;
};
Form bwd_form(int cols, int dtype)
{
    const int vec = dtype == CONV_F32 ? 4 : 8, most = 16 / vec, pieces = (cols + vec - 1) / vec;
    for (int lanes : {8, 16, 64, 256, 512}) {
        const int n = (pieces + lanes - 1) / lanes;
        if (n <= most && lanes < 512) return Form{lanes, n <= 1 ? 1 : n <= 2 ? 2 : 4};
        if (n <= most) return Form{lanes, most};
        if (n <= most * 3 / 2 && (lanes == 512 || (lanes >= 64 && vec == 8))) return Form{lanes, most * 3 / 2};
        if (n <= most * 2 && lanes == 512) return Form{lanes, most * 2};
    }
    return Form{0, 0};
}

// Forward: as above up to a wave; then waves as many as the row takes, up to 16, with 16 elements a lane (in 16 bits 32, where 16 waves
// would not do).  Against 4 or 16 waves, whose lanes were partly idle (us): 19660 x 2560 bf16 43 -> 35, 9830 x 5120 bf16 55 -> 35, codes alone
// 40 -> 28.  With few rows half of that a lane: 300 x 1536 bf16 3.7 -> 3.0; with many it costs, 12288 x 4096 bf16 34 -> 41.
struct FwdForm {
    int lanes, pieces, waves;
};
FwdForm fwd_form(int64_t rows, int cols, int dtype)
{
    const int vec = dtype == CONV_F32 ? 4 : 8, most = 16 / vec, pieces = (cols + vec - 1) / vec;
    for (int lanes : {8, 16, 64}) {
        const int n = (pieces + lanes - 1) / lanes;
        if (n <= most) return {lanes, n <= 1 ? 1 : n <= 2 ? 2 : 4, 0};
    }
    for (int n = rows <= 2 * kCUs ? most / 2 : most; n <= 4; n *= 2)
        if ((pieces + 64 * n - 1) / (64 * n) <= 16) return {0, n, (pieces + 64 * n - 1) / (64 * n)};
    return {0, 0, 0};
}

template <int DT, int G, int NV, int MODE>
void fwd_launch(const NormArgs& a, int waves, hipStream_t s)
{
    const int rows = G ? 256 / G : 1;
    // a workgroup a row: no more than the registers leave room for at once (5225 x 9632 bf16 56 us with 32 waves a CU, 35 with 20); where
    // workgroups are small a few more do no harm (196608 x 256 bf16 34 us with 8, 36 with 6)
    const int room = G || MODE == QUANT_ONLY || NV * (16 / (int)dtype_size(DT)) < 16 ? 32 : DT == CONV_F32 ? 20 : 24;
    const int64_t blocks = std::min<int64_t>((a.rows + rows - 1) / rows, kCUs * (room / waves));
    hipLaunchKernelGGL((norm_fwd_rows<DT, G, NV, MODE>), dim3((unsigned)blocks), dim3(64 * waves), 0, s, a);
}

template <int DT, int G, int MODE>
void fwd_pieces(const NormArgs& a, int nv, int waves, hipStream_t s)
{
    if (nv == 1) fwd_launch<DT, G, 1, MODE>(a, waves, s);
    else if (nv == 2) fwd_launch<DT, G, 2, MODE>(a, waves, s);
    else if constexpr (DT == CONV_F32 || G == 0) fwd_launch<DT, G, 4, MODE>(a, waves, s);
}

template <int DT, int MODE>
hipError_t fwd(const NormArgs& a, hipStream_t s)
{
    const FwdForm f = fwd_form(a.rows, a.cols, DT);
    if (f.lanes == 8) fwd_pieces<DT, 8, MODE>(a, f.pieces, 4, s);
    else if (f.lanes == 16) fwd_pieces<DT, 16, MODE>(a, f.pieces, 4, s);
    else if (f.lanes == 64) fwd_pieces<DT, 64, MODE>(a, f.pieces, 4, s);
    else if (f.waves) fwd_pieces<DT, 0, MODE>(a, f.pieces, f.waves, s);
    else hipLaunchKernelGGL((norm_fwd_any<DT, MODE>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(1024), 0, s, a);
    return hipGetLastError();
}

template <int MODE>
hipError_t fwd_type(const NormArgs& a, int dtype, hipStream_t s)
{
    return dtype == CONV_F32 ? fwd<CONV_F32, MODE>(a, s) : dtype == CONV_F16 ? fwd<CONV_F16, MODE>(a, s) : fwd<CONV_BF16, MODE>(a, s);
}

// Workgroups of the backward kernel: one of 512 threads a CU, as a sum of 2 * cols floats each is written and read again, or two where a
// lane has one piece only (us with 256 / 512 workgroups: 16384 x 4096 bf16 79 / 84, 200704 x 192 fp32 95 / 101, 200704 x 64 fp16 42 / 31,
// 20000 x 384 fp16 23 / 19).  Rows of eight lanes go to twice as many of 256 threads (us with 512 / 256 threads: 24 x 64 fp32 3.6 / 3.1,
// 200 x 64 fp32 5.8 / 5.3, 1000 x 100 bf16 8.7 / 7.7, but 393216 x 128 bf16 57.2 / 57.9).
constexpr int bwd_threads(int lanes) { return lanes == 8 ? 256 : 512; }
int bwd_parts(int64_t rows, int cols, int dtype)
{
    const Form f = bwd_form(cols, dtype);
    if (!f.lanes) return (int)std::max<int64_t>(1, std::min<int64_t>(64, (rows + 15) / 16));
    const int here = bwd_threads(f.lanes) / f.lanes;
    return (int)std::max<int64_t>(1, std::min<int64_t>((f.pieces == 1 ? 2 * kCUs : kCUs) * (f.lanes == 8 ? 2 : 1), (rows + here - 1) / here));
}

template <int DT, int G, int NV>
void bwd_launch(const NormArgs& a, int parts, hipStream_t s)
{
    constexpr int NT = bwd_threads(G);
    const dim3 grid((unsigned)parts), block(NT);
    const bool dw = a.dgamma || a.dbeta;
    if (a.dx && dw) hipLaunchKernelGGL((norm_bwd_rows<DT, G, NV, NT, true, true>), grid, block, 0, s, a);
    else if (a.dx) hipLaunchKernelGGL((norm_bwd_rows<DT, G, NV, NT, true, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((norm_bwd_rows<DT, G, NV, NT, false, true>), grid, block, 0, s, a);
}

template <int DT, int G>
void bwd_pieces(const NormArgs& a, int nv, int parts, hipStream_t s)
{
    constexpr int MOST = DT == CONV_F32 ? 4 : 2;
    if (nv == MOST) bwd_launch<DT, G, MOST>(a, parts, s);
    if constexpr (G < 512) {
        if (nv == 1) bwd_launch<DT, G, 1>(a, parts, s);
        if (MOST == 4 && nv == 2) bwd_launch<DT, G, 2>(a, parts, s);
    }
    if constexpr (G == 512 || (G >= 64 && DT != CONV_F32))
        if (nv == MOST * 3 / 2) bwd_launch<DT, G, MOST * 3 / 2>(a, parts, s);
    if constexpr (G == 512)
        if (nv == MOST * 2) bwd_launch<DT, G, MOST * 2>(a, parts, s);
}

// 64 columns a workgroup where that makes a workgroup a CU, else 16: 423 sums of 2 x 384 columns took 4.7 us with 64.
// A launch holds less than 2^32 threads, 16 a column here: rows of more than 2^25 columns take several.
void join(const NormArgs& a, int parts, hipStream_t s)
{
    constexpr int64_t PORTION = (int64_t)1 << 26;
    const int64_t cols = 2 * (int64_t)a.cols;
    if (cols < 64 * kCUs) {
        hipLaunchKernelGGL((norm_dw_join<16>), dim3((unsigned)((cols + 15) / 16)), dim3(1024), 0, s, a, parts, 0);
        return;
    }
    for (int64_t from = 0; from < cols; from += PORTION)
        hipLaunchKernelGGL((norm_dw_join<64>), dim3((unsigned)((std::min(cols - from, PORTION) + 63) / 64)), dim3(1024), 0, s, a, parts, from);
}

template <int DT>
hipError_t bwd(const NormArgs& a, hipStream_t s)
{
    const Form f = bwd_form(a.cols, DT);
    const int parts = bwd_parts(a.rows, a.cols, DT);
    const bool dw = a.dgamma || a.dbeta;
    if (f.lanes) {
        if (f.lanes == 8) bwd_pieces<DT, 8>(a, f.pieces, parts, s);
        else if (f.lanes == 16) bwd_pieces<DT, 16>(a, f.pieces, parts, s);
        else if (f.lanes == 64) bwd_pieces<DT, 64>(a, f.pieces, parts, s);
        else if (f.lanes == 256) bwd_pieces<DT, 256>(a, f.pieces, parts, s);
        else bwd_pieces<DT, 512>(a, f.pieces, parts, s);
    } else {
        if (dw) hipLaunchKernelGGL((norm_dw_any<DT>), dim3((unsigned)((a.cols + 255) / 256), parts), dim3(256), 0, s, a);
        if (a.dx && a.rows) hipLaunchKernelGGL((norm_dx_any<DT>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(1024), 0, s, a);
    }
    if (dw && (parts > 1 || !f.lanes))
        join(a, parts, s);
    return hipGetLastError();
}

}  // namespace

size_t layernorm_bwd_workspace(int64_t rows, int cols, int dtype)
{
    const int parts = bwd_parts(rows, cols, dtype);
    return parts == 1 && bwd_form(cols, dtype).lanes ? 0 : (size_t)parts * 2 * cols * 4;
}

hipError_t launch_layernorm_fwd(NormArgs& a, int dtype, hipStream_t s)
{
    return a.q ? fwd_type<TO_CODES>(a, dtype, s) : fwd_type<TO_FLOAT>(a, dtype, s);
}

hipError_t launch_quantize_rows(QuantArgs& q, int dtype, hipStream_t s)
{
    NormArgs a = {};
    a.x = q.x, a.q = q.q, a.scale = q.scale, a.rows = q.rows, a.ldx = q.ldx, a.ldy = q.ldq, a.cols = q.cols;
    return fwd_type<QUANT_ONLY>(a, dtype, s);
}

hipError_t launch_layernorm_bwd(NormArgs& a, int dtype, hipStream_t s)
{
    return dtype == CONV_F32 ? bwd<CONV_F32>(a, s) : dtype == CONV_F16 ? bwd<CONV_F16>(a, s) : bwd<CONV_BF16>(a, s);
}

}  // namespace convfwd
