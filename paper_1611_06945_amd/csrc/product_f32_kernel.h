// Matrix products of fp32 operands on the 16-bit matrix units, the operands split into three bf16 parts each on their way to LDS.
//
//   C[m][n] = sum_k A(m, k) B(n, k),  either operand along the reduction or across it as in product_kernel.h
//
// x = x0 + x1 + x2 with 8 bits each holds all 24 bits of an fp32 value; of the nine products of parts the six that count are formed: 1 1, 0 2 and 2 0 first,
// then 0 1 and 1 0, then 0 0.  What is left out is below 2^-25 of a product.  Six products at the bf16 rate are 2.6 times as fast as the fp32 matrix
// instructions.  An element is split once for a workgroup: pieces of eight go from memory to registers and as three planes to
// LDS, so operands may start anywhere.  A stage has 32 of the reduction: 64 bytes of each row and plane (pieces at piece ^ (row / 4 % 4)), or 32 rows
// across.  There are two stages: the next one is split and written between the products of the present one, since splitting is as much vector work as half of
// the products' time and a workgroup that did one after the other took 2.1 us a step of 128 x 128, whose products are 0.64.  A piece is asked for anew as soon as it is
// split, a whole step ahead (8192 x 4096 x 4096: 1413 us with a step's loads behind its products, 1295 so; 2048 x 2048 x 2048 105
// and 96).  Sums leave 16 bytes a lane, a row's blocks one after the other, so that lines are written whole (1196 us, 230 TFLOP/s; 91; 10824 x 80 x 1600 with sum and residual 112 -> 86).  Bound by the splitting beside the products: vector work and matrix work are about as long, and two waves a SIMD overlap them in part.
#pragma once

#include "linear_common.h"
#include "split_products.h"

namespace convfwd {

template <int WT_, int WN_, int FT_, int FN_>
struct SplitTile {
    static constexpr int S = 2;  // stages
    static constexpr int WT = WT_, WN = WN_, FT = FT_, FN = FN_;
    static constexpr int BT = 16 * WT * FT, BN = 16 * WN * FN, NT = 64 * WT * WN, KE = 32;
    static constexpr int PLANE_A = BT * KE * 2, PLANE_B = BN * KE * 2;  // bytes of a plane of a stage
    static constexpr int STAGE = 3 * (PLANE_A + PLANE_B);
    static constexpr size_t LDS = S * STAGE + BN * 4;
    static constexpr int LA = BT * 4 / NT, LB = BN * 4 / NT;            // pieces of eight a thread
    static_assert(LA * NT == BT * 4 && LB * NT == BN * 4 && FN % 2 == 0, "whole loads");
};

template <typename T, int W, int L, bool ACROSS>
struct SplitOperand {
    typedef AnyPieces<float, T::NT, W, T::KE, L, ACROSS> Pieces;
    Pieces pieces;
    float held[L][8];  // the next step

    // pieces FROM .. TO - 1 of a step
    template <int FROM, int TO>
    __device__ __forceinline__ void load_whole()
    {
#pragma unroll
        for (int i = FROM; i < TO; ++i) pieces.load_whole(held[i], i);
    }
    template <int FROM, int TO>
    __device__ __forceinline__ void commit(char* lds, int plane)
    {
#pragma unroll
        for (int i = FROM; i < TO; ++i) {
            int row, piece;
            Pieces::place(i, row, piece);
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
    int64_t each;              // of the reduction, of each of the workgroups that share it: a multiple of the step
    int tiles_m, tiles_n, splits;
    float* partial;
};

template <typename T, bool A_ACROSS, bool B_ACROSS, bool PARTIAL>
__global__ __launch_bounds__(T::NT) void product_f32_kernel(SplitArgs g, LinearOut e)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wt = wave % T::WT, wn = wave / T::WT;
    int tile, tm, tn;
    const int share = share_of_block(g.splits, tile);
    place_of_tile(tile, g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * T::BT, n0 = (int64_t)tn * T::BN;
    const int64_t k0 = share * g.each, k1 = min(k0 + g.each, g.K);

    SplitOperand<T, T::BT, T::LA, A_ACROSS> a;
    SplitOperand<T, T::BN, T::LB, B_ACROSS> b;
    a.pieces.begin(g.a, g.lda, k1, m0, g.M, k0);
    b.pieces.begin(g.b, g.ldb, k1, n0, g.N, k0);
    float* const bias = (float*)(smem + T::S * T::STAGE);
    if constexpr (!PARTIAL) LinearEpi<CONV_F32>::prepare(e, bias, n0, b.pieces.here, T::BN, T::NT);

    f32x4 acc[T::FN][T::FT];
#pragma unroll
    for (int i = 0; i < T::FN; ++i)
#pragma unroll
        for (int j = 0; j < T::FT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    auto commit = [&](char* stage, auto part) {  // part of FT
        constexpr int P = decltype(part)::value;
        a.template commit<T::LA * P / T::FT, T::LA * (P + 1) / T::FT>(stage, T::PLANE_A);
        b.template commit<T::LB * P / T::FT, T::LB * (P + 1) / T::FT>(stage + 3 * T::PLANE_A, T::PLANE_B);
    };
    // The products of the step in stage `buf`; between them the step that the registers hold, if there is one, is split and goes to the other
    // stage, and each of its pieces may be asked for anew for the step after it.
    int buf = 0;
    auto step = [&](auto load, bool more) {
        const char *const at_a = smem + buf * T::STAGE, *const at_b = at_a + 3 * T::PLANE_A;
        char* const next = smem + (buf ^ 1) * T::STAGE;
        u32x4 bv[T::FN][3];
#pragma unroll
        for (int i = 0; i < T::FN; ++i)
#pragma unroll
            for (int q = 0; q < 3; ++q) bv[i][q] = b.fragment(at_b + q * T::PLANE_B, wn * T::FN + i);
        count_to<T::FT>([&](auto part) {
            constexpr int j = decltype(part)::value;
            u32x4 av[3];
#pragma unroll
            for (int q = 0; q < 3; ++q) av[q] = a.fragment(at_a + q * T::PLANE_A, wt * T::FT + j);
            if (more) commit(next, part);
            load(part);
            constexpr int PA[6] = {1, 0, 2, 0, 1, 0}, PB[6] = {1, 2, 0, 1, 0, 0};
#pragma unroll
            for (int t = 0; t < 6; ++t)
#pragma unroll
                for (int i = 0; i < T::FN; ++i) acc[i][j] = multiply16<CONV_BF16>(bv[i][PB[t]], av[PA[t]], acc[i][j]);
        });
        buf ^= 1;
    };

    const int steps = (int)((k1 - k0 + T::KE - 1) / T::KE);
    a.pieces.load(a.held), b.pieces.load(b.held);
    a.pieces.clear(a.held), b.pieces.clear(b.held);
    count_to<T::FT>([&](auto p) { commit(smem, p); });
    // Whole steps: loads without a branch (behind one that may load or not a wave waits for all that is on its way), a step ahead.
    const int whole = min(a.pieces.whole(), b.pieces.whole()) - 1;
    auto load_whole = [&](auto part) {
        constexpr int P = decltype(part)::value;
        a.template load_whole<T::LA * P / T::FT, T::LA*(P + 1) / T::FT>();
        b.template load_whole<T::LB * P / T::FT, T::LB*(P + 1) / T::FT>();
    };
    int k = 0;
    if (whole > 0) {
        count_to<T::FT>(load_whole);
        a.pieces.advance(), b.pieces.advance();
        __syncthreads();
        for (; k < whole; ++k) {
            a.pieces.keep(), b.pieces.keep();
            step(load_whole, true);
            a.pieces.advance(), b.pieces.advance();
            __syncthreads();
        }
    } else {
        a.pieces.load(a.held), b.pieces.load(b.held);
        __syncthreads();
    }
    for (; k < steps; ++k) {
        if (k + 1 < steps) a.pieces.clear(a.held), b.pieces.clear(b.held);
        step([](auto) {}, k + 1 < steps);
        a.pieces.load(a.held), b.pieces.load(b.held);  // (past the last step: nothing)
        __syncthreads();
    }

    // a lane has four n in a row, 16 bytes; the blocks of a row one after the other
    float columns[T::FN][4];
    if constexpr (!PARTIAL) {
#pragma unroll
        for (int i = 0; i < T::FN; ++i) __builtin_memcpy(columns[i], bias + (wn * T::FN + i) * 16 + (lane >> 4) * 4, 16);
    }
#pragma unroll
    for (int j = 0; j < T::FT; ++j) {
        const int ml = (wt * T::FT + j) * 16 + (lane & 15);
        const int64_t m = g.m_first + m0 + ml;
#pragma unroll
        for (int i = 0; i < T::FN; ++i) {
            const int nl = (wn * T::FN + i) * 16 + (lane >> 4) * 4;
            if (ml < a.pieces.here && nl < b.pieces.here) {
                float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                const int have = min(4, b.pieces.here - nl);
                if constexpr (PARTIAL) put_pieces<CONV_F32, 4>(g.partial, ((int64_t)share * g.M + m) * g.N + n0 + nl, v, have);
                else LinearEpi<CONV_F32>::finish(ProductArgs(), e, v, m, n0 + nl, have, columns[i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

}  // namespace convfwd
