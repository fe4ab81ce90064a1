// Matrix products of fp32 operands on the 16-bit matrix units, the operands split into three bf16 parts each on their way to LDS.
//
//   C[m][n] = sum_k A(m, k) B(n, k),  either operand along the reduction or across it as in product_kernel.h
//
// x = x0 + x1 + x2 with 8 bits each holds all 24 bits of an fp32 value; of the nine products of parts the six that count are formed: 1 1, 0 2 and 2 0 first,
// then 0 1 and 1 0, then 0 0.  What is left out is below 2^-25 of a product.  Six products at the bf16 rate are 2.6 times as fast as the fp32 matrix
// instructions.  An element is split once for a workgroup: pieces of eight go from memory to registers, one step ahead, and as three planes to
// LDS, so operands may start anywhere.  A stage has 32 of the reduction: 64 bytes of each row and plane (pieces at piece ^ (row / 4 % 4)), or 32 rows
// across.  One stage only, so that two or three workgroups a CU fill each other's waits.
#pragma once

#include "linear_common.h"
#include "split_products.h"

namespace convfwd {

template <int WT_, int WN_, int FT_, int FN_>
struct SplitTile {
    static constexpr int WT = WT_, WN = WN_, FT = FT_, FN = FN_;
    static constexpr int BT = 16 * WT * FT, BN = 16 * WN * FN, NT = 64 * WT * WN, KE = 32;
    static constexpr int PLANE_A = BT * KE * 2, PLANE_B = BN * KE * 2;  // bytes of a plane of a stage
    static constexpr size_t LDS = 3 * (PLANE_A + PLANE_B) + BN * 4;
    static constexpr int LA = BT * 4 / NT, LB = BN * 4 / NT;            // pieces of eight a thread
    static_assert(LA * NT == BT * 4 && LB * NT == BN * 4 && FN % 2 == 0, "whole loads");
};

template <typename T, int W, int L, bool ACROSS>
struct SplitOperand {
    const float* from;  // the tile's first element of the next step
    int64_t ld, left;   // left: of the reduction
    int here;
    float held[L][8];

    static __device__ __forceinline__ void place(int i, int& row, int& piece)
    {
        const int p = i * T::NT + (int)threadIdx.x;
        row = ACROSS ? p / (W / 8) : p / 4, piece = ACROSS ? p % (W / 8) : p % 4;
    }
    __device__ __forceinline__ void begin(const float* p, int64_t stride, int64_t K, int64_t first, int64_t all, int64_t k0)
    {
        ld = stride, left = K - k0;
        here = (int)min((int64_t)W, all - first);
        from = p + (ACROSS ? first + k0 * stride : first * stride + k0);
    }
    __device__ __forceinline__ void load()
    {
        const bool whole = here == W && left >= T::KE;
#pragma unroll
        for (int i = 0; i < L; ++i) {
            int row, piece;
            place(i, row, piece);
            const float* p = from + row * ld + piece * 8;
            const int64_t n = ACROSS ? (row < left ? here - piece * 8 : 0) : (row < here ? left - piece * 8 : 0);
            if (whole || n >= 8) {
                __builtin_memcpy(held[i], p, 32);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) held[i][j] = j < n ? p[j] : 0.0f;
            }
        }
        from += ACROSS ? T::KE * ld : (int64_t)T::KE;
        left -= T::KE;
    }
    __device__ __forceinline__ void commit(char* lds, int plane) const
    {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            int row, piece;
            place(i, row, piece);
            const Split3 s = split3(held[i]);
            char* to = lds + (ACROSS ? row * (W * 2) + (piece ^ across_swizzle<W>(row)) * 16 : row * 64 + ((piece ^ ((row >> 2) & 3)) << 4));
#pragma unroll
            for (int q = 0; q < 3; ++q) *(uint4*)(to + q * plane) = s.p[q];
        }
    }
    static __device__ __forceinline__ u32x4 fragment(const char* lds, int block)
    {
        const int lane = threadIdx.x & 63;
        if constexpr (ACROSS) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const int k = (lane >> 4) * 8 + ((lane & 15) >> 2);
            const char* p = lds + k * (W * 2) + ((block * 2) ^ across_swizzle<W>(k)) * 16 + (lane & 3) * 8;
            union {
                s16x4 h[2];
                u32x4 v;
            } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * W * 2));
            return u.v;
        } else {
            return *(const u32x4*)(lds + block * 1024 + (lane & 15) * 64 + (((lane >> 4) ^ ((lane >> 2) & 3)) << 4));
        }
    }
};

struct SplitArgs {
    const float *a, *b;
    int64_t lda, ldb;
    int64_t M, N, K, m_first;
    int64_t each;              // of the reduction, of a workgroup that shares it with others (gridDim.z): a multiple of the step
    int tiles_m, tiles_n;
    float* partial;
};

template <typename T, bool A_ACROSS, bool B_ACROSS, bool PARTIAL>
__global__ __launch_bounds__(T::NT) void product_f32_kernel(SplitArgs g, LinearOut e)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wt = wave % T::WT, wn = wave / T::WT;
    int tm, tn;
    tile_of_block(g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * T::BT, n0 = (int64_t)tn * T::BN;
    const int64_t k0 = blockIdx.z * g.each, k1 = min(k0 + g.each, g.K);

    SplitOperand<T, T::BT, T::LA, A_ACROSS> a;
    SplitOperand<T, T::BN, T::LB, B_ACROSS> b;
    a.begin(g.a, g.lda, k1, m0, g.M, k0);
    b.begin(g.b, g.ldb, k1, n0, g.N, k0);
    char *const lds_a = smem, *const lds_b = smem + 3 * T::PLANE_A;
    float* const bias = (float*)(smem + 3 * (T::PLANE_A + T::PLANE_B));
    if constexpr (!PARTIAL) LinearEpi<CONV_F32>::prepare(e, bias, n0, b.here, T::BN, T::NT);

    f32x4 acc[T::FN][T::FT];
#pragma unroll
    for (int i = 0; i < T::FN; ++i)
#pragma unroll
        for (int j = 0; j < T::FT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    a.load(), b.load();
    for (int64_t k = k0; k < k1; k += T::KE) {
        __syncthreads();  // the stage has been read
        a.commit(lds_a, T::PLANE_A), b.commit(lds_b, T::PLANE_B);
        __syncthreads();
        if (k + T::KE < k1) a.load(), b.load();
        u32x4 bv[T::FN][3];
#pragma unroll
        for (int i = 0; i < T::FN; ++i)
#pragma unroll
            for (int q = 0; q < 3; ++q) bv[i][q] = b.fragment(lds_b + q * T::PLANE_B, wn * T::FN + i);
#pragma unroll
        for (int j = 0; j < T::FT; ++j) {
            u32x4 av[3];
#pragma unroll
            for (int q = 0; q < 3; ++q) av[q] = a.fragment(lds_a + q * T::PLANE_A, wt * T::FT + j);
            constexpr int PA[6] = {1, 0, 2, 0, 1, 0}, PB[6] = {1, 2, 0, 1, 0, 0};
#pragma unroll
            for (int t = 0; t < 6; ++t)
#pragma unroll
                for (int i = 0; i < T::FN; ++i) acc[i][j] = multiply16<CONV_BF16>(bv[i][PB[t]], av[PA[t]], acc[i][j]);
        }
    }

    // as in product_kernel: eight n in a row for each lane
    const int grp = lane >> 4;
#pragma unroll
    for (int i = 0; i < T::FN; i += 2) {
        const int nl = (wn * T::FN + i) * 16 + (grp & 1) * 16 + (grp >> 1) * 8;
#pragma unroll
        for (int j = 0; j < T::FT; ++j) {
            const int ml = (wt * T::FT + j) * 16 + (lane & 15);
            float v[8];
            eight_in_a_row(acc[i][j], acc[i + 1][j], v);
            if (ml < a.here && nl < b.here) {
                const int have = min(8, b.here - nl);
                const int64_t m = g.m_first + m0 + ml;
                if constexpr (PARTIAL) put8<CONV_F32>(g.partial, ((int64_t)blockIdx.z * g.M + m) * g.N + n0 + nl, v, have);
                else LinearEpi<CONV_F32>::finish(ProductArgs(), e, v, m, n0 + nl, have, bias + nl);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

}  // namespace convfwd
