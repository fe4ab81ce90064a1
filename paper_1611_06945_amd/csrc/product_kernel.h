// Matrix products in 16 bits with fp32 sums, and what is done with a tile of sums before it leaves: the core of the linear layers, their
// gradients and the Newton-Schulz update.
//
//   C[m][n] = sum_k A(m, k) B(n, k)
//
// Either operand lies along the reduction (ALONG: A(m, k) at m ld + k, as x and w do forward) or across it (ACROSS: at k ld + m, as w does in
// the gradient of x, and both do in the gradient of w).  Tiles of BT x BN, both operands staged through LDS in steps of 64 of the
// reduction (128 bytes), multiplied by 16x16x32 matrix instructions, with n along the registers: a lane has 4 consecutive n of row m = lane % 16.
//   * ALONG: a stage holds 128 bytes of each row, its eight 16-byte pieces at piece ^ (row / 2 % 8), so that the 16 lanes that LDS serves
//     together read 16 different groups of four banks.
//   * ACROSS: a stage holds 64 rows of BT elements; an operand is read by two transposing LDS reads of 4 k x 16 m, each lane 8 bytes.  Such a
//     read of a wave touches 32 bytes of 16 rows; pairs of pieces are stored at pair ^ swizzle(k), so that 8 rows lie in all 64 banks.
//   * DIRECT: loads that write LDS themselves, from operands whose rows start on 16 bytes; what is past an operand's end is read as zeros by
//     the bounds check of the buffer descriptor, which moves along with the reduction, so that offsets stay below 2^31 however long it is.  A row's
//     bytes past K belong to what follows and are cleared in both operands on the last step.  Otherwise pieces go
//     through registers, from any address, and their ends are cleared on the way.
//   * Operands may be sums of two planes, high and low (PL = 2), of which a step multiplies low x high, high x low and high x high.
//   * PARTS: A alone is a sum of two planes, what the storage type holds of it and what is left (Parts).  The reduction is gone through twice, for the low
//     plane first, whose sums are scaled before those of the high one are added to them: LDS has no room for a third plane beside the largest tiles.  (The
//     code of both passes is laid out: in a loop the tiles of 256 x 256 spilled some 30 registers.)
// Bound by the matrix units and LDS together: a step of a tile of 256 x 256 takes 2048 clocks of products and 2048 of LDS, 1536 reading and 512 written to, so waves of
// 64 x 128 with two a SIMD, each's products between the reads of its next operands.  8192 x 4096 x 8192 bf16 with GELU and the sum kept 475 to 483 us, 1.14 PFLOP/s, matrix
// units busy 52 % of the clocks (the end of a tile, 45 us in all, has none); four waves of 128 x 128 with one a SIMD took 141 us for 4096 x 4096 x 4096 where this takes 100.
#pragma once

#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "rows_common.h"

namespace convfwd {

typedef __attribute__((address_space(3))) void lds_void_t;

template <int N, typename F>
__device__ __forceinline__ void count_to(F f)
{
    if constexpr (N > 0) {
        count_to<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

template <int WT_, int WN_, int FT_, int FN_, int S_, int PL_ = 1>
struct ProductTile {
    static constexpr int PL = PL_;  // planes
    static constexpr int WT = WT_, WN = WN_, FT = FT_, FN = FN_, S = S_;  // waves and 16-wide blocks a wave, along m and n; stages
    static constexpr int BT = 16 * WT * FT, BN = 16 * WN * FN, NT = 64 * WT * WN;
    static constexpr int KB = 128, KE = KB / 2;  // of a step, bytes and elements
    static constexpr int PLANE_A = BT * KB, PLANE_B = BN * KB, STAGE = PL * (PLANE_A + PLANE_B);
    static constexpr size_t LDS = (size_t)S * STAGE + BN * 4;
    static constexpr int LA = BT * 8 / NT, LW = BN * 8 / NT;  // 16-byte loads a thread and stage
    static constexpr int H = FT > 4 ? 2 : 1, HB = FT / H;     // the blocks of m go in H portions
    static_assert(S >= 2, "a stage to multiply, one to load");
    static_assert(LA * NT == BT * 8 && LW * NT == BN * 8 && FN % 2 == 0 && HB * H == FT, "whole loads and portions");
};

// Where pair p of 16-byte pieces of row k is stored in a stage of an operand that lies across the reduction: 2 p ^ this.
template <int W>
__device__ __forceinline__ int across_swizzle(int k)
{
    return W % 128 == 0 ? ((k & 3) | ((k >> 3) & 1) << 2) * 2 : (((k >> 1) & 1) | ((k >> 3) & 1) << 1) * 2;
}

// The first `n` elements of 8 (n may be <= 0 or >= 8), the others zero.
__device__ __forceinline__ u32x4 first_elems(u32x4 v, int n)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int have = n - 2 * i;
        v[i] = have >= 2 ? v[i] : have <= 0 ? 0u : v[i] & 0xFFFFu;
    }
    return v;
}

template <int DT>
__device__ __forceinline__ f32x4 multiply16(u32x4 b, u32x4 a, f32x4 c)
{
    if constexpr (DT == CONV_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, b), __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
}

// Pieces of eight elements from any address to registers, KE of the reduction a step, L pieces a thread.  Loads have no branch around them that lanes take apart: a wave
// would wait there for all its loads, and a step take a trip to memory.  Instead a lane without a piece reads another one's, and what a
// piece holds past the reduction's end is cleared where it is used.  Only a step in which a piece would pass the end of the whole operand
// loads element by element.
template <typename E, int NT, int W, int KE, int L, bool ACROSS>
struct AnyPieces {
    const E* from;  // the tile's first element of the next step
    int64_t ld, left, used;  // left: of the reduction, for load; used: for clear
    int here;                // rows (ALONG) or columns (ACROSS) of the tile that exist
    bool last;               // ALONG: whether nothing follows the tile's last row; ACROSS: whether a piece passes the last column
    int64_t off[L];

    static __device__ __forceinline__ void place(int i, int& row, int& piece)
    {
        const int p = i * NT + (int)threadIdx.x;
        row = ACROSS ? p / (W / 8) : p / (KE / 8), piece = ACROSS ? p % (W / 8) : p % (KE / 8);
    }
    __device__ __forceinline__ void begin(const E* p, int64_t stride, int64_t K, int64_t first, int64_t all, int64_t k0)
    {
        ld = stride, left = used = K - k0;
        here = (int)min((int64_t)W, all - first);
        last = ACROSS ? (here & 7) != 0 : first + here >= all || K < 8;
        from = p + (ACROSS ? first + k0 * stride : first * stride + k0);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            int row, piece;
            place(i, row, piece);
            off[i] = ACROSS ? row * ld + (piece * 8 < here ? piece * 8 : 0) : min(row, here - 1) * ld + piece * 8;
        }
    }
    // Steps from here on that load whole pieces.  (ACROSS: eight more rows hold the seven elements that a piece may pass its row's last column
    // by, however short they are)
    __device__ __forceinline__ int whole() const { return (int)min(max((left - (ACROSS && last ? 8 : 0)) / KE, (int64_t)0), (int64_t)INT_MAX); }
    // piece i of one of those; advance() after all of its pieces
    __device__ __forceinline__ void load_whole(E (&to)[8], int i) { __builtin_memcpy(to, from + off[i], 8 * sizeof(E)); }
    __device__ __forceinline__ void advance()
    {
        from += ACROSS ? KE * ld : (int64_t)KE;
        left -= KE;
    }
    __device__ __forceinline__ void load(E (&to)[L][8])
    {
        if (left >= KE + (ACROSS && last ? 8 : 0)) {
#pragma unroll
            for (int i = 0; i < L; ++i) load_whole(to[i], i);
        } else if (left > 0) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                int row, piece;
                place(i, row, piece);
                if (!last) {
                    // (ALONG: a piece that passes its row's end goes on in the next row)
                    const int64_t at = ACROSS ? min((int64_t)row, left - 1) * ld + (piece * 8 < here ? piece * 8 : 0)
                                              : min(row, here - 1) * ld + (piece * 8 < left ? piece * 8 : 0);
                    __builtin_memcpy(to[i], from + at, 8 * sizeof(E));
                } else {
                    const E* p = from + row * ld + piece * 8;
                    const int64_t n = ACROSS ? (row < left ? here - piece * 8 : 0) : (row < here ? left - piece * 8 : 0);
#pragma unroll
                    for (int j = 0; j < 8; ++j) to[i][j] = j < n ? p[j] : (E)0;
                }
            }
        }
        advance();
    }
    // a step of whole pieces within the reduction
    __device__ __forceinline__ void keep() { used -= KE; }
    // what is past the reduction's end becomes zeros; this or keep() once for each load, in their order
    __device__ __forceinline__ void clear(E (&v)[L][8])
    {
        if (used < KE) {
#pragma unroll
            for (int i = 0; i < L; ++i) {
                int row, piece;
                place(i, row, piece);
                const int64_t n = ACROSS ? (row < used ? 8 : 0) : used - piece * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = j < n ? v[i][j] : (E)0;
            }
        }
        used -= KE;
    }
};

// 16 bytes a lane from offset `off` of a descriptor to LDS, the wave's 1024 bytes from `to`.  It is the instruction of
// __builtin_amdgcn_raw_ptr_buffer_load_lds, written out because the compiler lets no transposing LDS read (a builtin that may read anything)
// pass such a builtin without waiting for all of them: a step's loads would have a quarter of the step to arrive.  It has no
// output register; what it writes is waited for by count and barrier below, and its operands are read when it is issued.
__device__ __forceinline__ void load_to_lds(u32x4 r, uint32_t to, uint32_t off)
{
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to), "v"(off), "s"(r));
}

// The matrix operand of block `block` (16 wide) for half s of a stage of 64 of the reduction.
template <int W, bool ACROSS>
__device__ __forceinline__ u32x4 fragment_of(const char* lds, int block, int s)
{
    const int lane = threadIdx.x & 63;
    if constexpr (ACROSS) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const int k = (lane >> 4) * 8 + ((lane & 15) >> 2);
        const char* p = lds + (s * 32 + k) * (W * 2) + ((block * 2) ^ across_swizzle<W>(k)) * 16 + (lane & 3) * 8;
        union {
            s16x4 h[2];
            u32x4 v;
        } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * W * 2));
        return u.v;
    } else {
        return *(const u32x4*)(lds + block * 2048 + (lane & 15) * 128 + (((s * 4 + (lane >> 4)) ^ ((lane >> 1) & 7)) << 4));
    }
}
// Where a piece of such a stage lies: 16-byte piece `piece` of row `row` (of the operand ALONG, of the reduction ACROSS).
template <int W, bool ACROSS>
__device__ __forceinline__ int swizzled(int row, int piece)
{
    return ACROSS ? piece ^ across_swizzle<W>(row) : piece ^ ((row >> 1) & 7);
}

// One operand of a tile.  W: its width (BT or BN), L: pieces a thread and stage.
template <typename T, int W, int L, bool ACROSS, bool DIRECT>
struct Operand {
    int64_t ld, plane;
    int here;              // rows (ALONG) or columns (ACROSS) of the tile that exist
    const uint16_t* from;  // the next step, first plane
    int64_t left;          // bytes from there to the operand's end, in whole pieces
    uint32_t off[L];

    __device__ __forceinline__ void begin(const uint16_t* p, int64_t stride, int64_t plane_, int64_t K, int64_t first, int64_t all, int64_t k0)
    {
        ld = stride, plane = plane_;
        here = (int)min((int64_t)W, all - first);
        from = p + (ACROSS ? first + k0 * ld : first * ld + k0);
        // (the rows start on 16 bytes, so what the last piece holds past the end lies in the same 16 bytes as an element)
        left = ((ACROSS ? (K - 1 - k0) * ld + here : (here - 1) * ld + (K - k0)) * 2 + 15) & ~(int64_t)15;
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int p = i * T::NT + (int)threadIdx.x, row = ACROSS ? p / (W / 8) : p / 8, piece = ACROSS ? p % (W / 8) : p % 8;
            off[i] = (uint32_t)row * (uint32_t)(stride * 2) + swizzled<W, ACROSS>(row, piece) * 16;
        }
    }
    __device__ __forceinline__ void advance()
    {
        const int64_t by = ACROSS ? T::KE * ld : T::KE;
        from += by;
        left -= by * 2;
    }
    // the next step to the stage at `lds`, plane behind plane (no step: nothing but zeros)
    __device__ __forceinline__ void load(char* lds, bool step)
    {
        const uint32_t bytes = !step || left <= 0 ? 0u : (uint32_t)min(left, (int64_t)0x7FFFFFF0);
#pragma unroll
        for (int q = 0; q < T::PL; ++q) {
            const uint64_t at = (uint64_t)(uintptr_t)(from + q * plane);
            const u32x4 r = {(uint32_t)at, (uint32_t)(at >> 32), bytes, 0x00020000u};
            const uint32_t to = (uint32_t)(uintptr_t)(lds_void_t*)lds + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024 + q * (W * T::KB);
#pragma unroll
            for (int i = 0; i < L; ++i) load_to_lds(r, to + i * T::NT * 16, off[i]);
        }
    }
    static __device__ __forceinline__ u32x4 fragment(const char* lds, int block, int s) { return fragment_of<W, ACROSS>(lds, block, s); }
};

// ... that may start anywhere, through registers, of one plane
template <typename T, int W, int L, bool ACROSS>
struct Operand<T, W, L, ACROSS, false> {
    typedef AnyPieces<uint16_t, T::NT, W, T::KE, L, ACROSS> Pieces;
    // Steps on their way: a step of small tiles takes a fraction of a trip to memory (64 x 64 with 1 and 4: the gradient of x of 777 x 1283 x 1001 25.6 and 18.6 us;
    // 128 x 128 with 1, 2 and 4: that of w 25.7, 21.3 and 23.2 us, for the registers that two workgroups a CU have).
    static constexpr int D = L == 1 ? 4 : 2;
    Pieces pieces;
    int here;
    uint16_t held[D][L][8];

    __device__ __forceinline__ void begin(const uint16_t* p, int64_t stride, int64_t, int64_t K, int64_t first, int64_t all, int64_t k0)
    {
        pieces.begin(p, stride, K, first, all, k0);
        here = pieces.here;
    }
    template <int S>
    __device__ __forceinline__ void load_whole()
    {
#pragma unroll
        for (int i = 0; i < L; ++i) pieces.load_whole(held[S][i], i);
        pieces.advance();
    }
    template <int S, bool WHOLE>
    __device__ __forceinline__ void commit(char* lds)
    {
        if constexpr (WHOLE) pieces.keep();
        else pieces.clear(held[S]);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            int row, piece;
            Pieces::place(i, row, piece);
            uint4 v;
            __builtin_memcpy(&v, held[S][i], 16);
            *(uint4*)(lds + (row * (ACROSS ? W / 8 : 8) + swizzled<W, ACROSS>(row, piece)) * 16) = v;
        }
    }
    static __device__ __forceinline__ u32x4 fragment(const char* lds, int block, int s) { return fragment_of<W, ACROSS>(lds, block, s); }
};

// A value v in two elements of a 16-bit type: high of v HIGH, low of what is left of that times LOW.  bf16 has fp32's exponents and needs neither
// factor.  fp16: half of the largest value times the largest slope of an activation, 1.13, is no infinity yet, and what is left of a value that fp16 holds as a denormal
// number or not at all is kept down to 2^-36.
template <int DT>
struct Parts {
    static constexpr float HIGH = DT == CONV_F16 ? 0.5f : 1.0f, LOW = DT == CONV_F16 ? 0x1p11f : 1.0f;
    static __device__ __forceinline__ void split(const float (&v)[8], float (&high)[8], float (&low)[8])
    {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float x = v[k] * HIGH;
            high[k] = Prec<DT>::to_f32(Prec<DT>::from_f32(x));
            low[k] = fabsf(high[k]) < INFINITY ? (x - high[k]) * LOW : 0.0f;  // an infinity stays one; a NaN is in the high part
        }
    }
};

struct ProductArgs {
    const uint16_t *a, *b;
    int64_t lda, ldb;             // of operands, in elements of 16 bits
    int64_t plane_a, plane_b;     // distance of an operand's planes
    int64_t M, N, K;
    int64_t m_first;              // what the first row of these M is in the whole product
    int ksteps, each, splits;     // steps of the reduction, and of each of the workgroups that share it
    int64_t batch_a, batch_b;     // distances of the batch's matrices (gridDim.y)
    int tiles_m, tiles_n;
    float* partial;               // sums of the workgroups that share a reduction, [splits][M][N]
};

// Consecutive workgroups go to different XCDs: each XCD takes a run of tiles.
__device__ __forceinline__ int tile_in_order()
{
    const int total = gridDim.x, q = total / 8, r = total % 8, x = blockIdx.x % 8, i = blockIdx.x / 8;
    return x * q + min(x, r) + i;
}
// Where `splits` workgroups share a tile's reduction, consecutive workgroups take different shares of it, so that an XCD has all tiles of its
// shares and reads only those parts of the operands (2048 x 1024 x 50257 in shares of 8: 260 us with the tiles dealt to the XCDs).
__device__ __forceinline__ int share_of_block(int splits, int& tile)
{
    if (splits == 1) {
        tile = tile_in_order();
        return 0;
    }
    tile = blockIdx.x / splits;
    return blockIdx.x % splits;
}
// ... in bands of eight tiles of n
__device__ __forceinline__ void place_of_tile(int tile, int tiles_m, int tiles_n, int& tm, int& tn)
{
    const int band = tile / (8 * tiles_m), in_band = tile - band * 8 * tiles_m;
    const int width = min(8, tiles_n - band * 8);
    tn = band * 8 + in_band % width, tm = in_band / width;
}
// ... of those with n >= m only: row tm has the tiles tm .. tiles - 1
__device__ __forceinline__ void tile_above_diagonal(int tile, int tiles, int& tm, int& tn)
{
    tm = 0;
    for (int left = tiles; tile >= left; --left) tile -= left, ++tm;
    tn = tm + tile;
}

// A lane has four n 4 (lane / 16) .. of a block and m = lane % 16 of a block of rows.  Neighbouring groups of 16 lanes trade between two
// blocks of n, so that a lane has eight n in a row: the groups 0 .. 3 those of the first block from 0, of the second from 0, of the first
// from 8, of the second from 8.
__device__ __forceinline__ void eight_in_a_row(const f32x4& first, const f32x4& second, float (&v)[8])
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float here = first[r], there = second[r];  // (a cast of a vector's element itself takes the first one)
        const auto two = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, here), __builtin_bit_cast(uint32_t, there), false, false);
        v[r] = __builtin_bit_cast(float, (uint32_t)two[0]), v[4 + r] = __builtin_bit_cast(float, (uint32_t)two[1]);
    }
}

// Epi: what becomes of the sums.  symmetric: only the tiles with n >= m are formed.
template <int DT, typename T, bool A_ACROSS, bool B_ACROSS, bool DIRECT, typename Epi, bool PARTS>
__global__ __launch_bounds__(T::NT) void product_kernel(ProductArgs g, typename Epi::Args e)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave % T::WT, wn = wave / T::WT;

    int tile, tm, tn;
    const int share = share_of_block(g.splits, tile);
    if constexpr (Epi::SYMMETRIC) tile_above_diagonal(tile, g.tiles_m, tm, tn);
    else place_of_tile(tile, g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * T::BT, n0 = (int64_t)tn * T::BN;
    const int ks0 = share * g.each, ks1 = min(ks0 + g.each, g.ksteps);

    Operand<T, T::BT, T::LA, A_ACROSS, DIRECT> a;
    Operand<T, T::BN, T::LW, B_ACROSS, DIRECT> b;
    auto begin = [&](int64_t plane) {
        a.begin(g.a + blockIdx.y * g.batch_a + plane, g.lda, g.plane_a, g.K, m0, g.M, (int64_t)ks0 * T::KE);
        b.begin(g.b + blockIdx.y * g.batch_b, g.ldb, g.plane_b, g.K, n0, g.N, (int64_t)ks0 * T::KE);
    };
    begin(PARTS ? g.plane_a : 0);
    float* const bias = (float*)(smem + T::S * T::STAGE);
    Epi::prepare(e, bias, n0, b.here, T::BN, T::NT);

    const int steps = ks1 - ks0;
    f32x4 acc[T::FN][T::FT];
#pragma unroll
    for (int i = 0; i < T::FN; ++i)
#pragma unroll
        for (int j = 0; j < T::FT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // Two planes: the products with a low one add up apart, in small tiles also those of a step's second half, so that the large sums are of a third or a sixth as many
    // terms: after six of the steps of orthogonal.hip fp32 matrices of 24 x 3168 are off by 1.9e-6 of the norm, with one sum 4.6e-6 (in fp32 products 1.6e-6).  (In tiles of 128 x
    // 128 a third sum takes 5 to 8 % more time; the larger matrices that take those are off by 0.4 of what fp32 products are with two.)
    constexpr bool APART = T::PL == 2, HALVES = APART && T::FN * T::FT <= 2;
    f32x4 apart[HALVES ? 2 : 1][APART ? T::FN : 1][APART ? T::FT : 1] = {};

    u32x4 av[2][T::PL][T::HB], bv[2][T::PL][T::FN];
    // The operands of phase p of a stage (half p / H, portion p % H of the rows) to the registers of its parity.
    auto fetch = [&](int buf, auto phase) {
        constexpr int p = decltype(phase)::value, s = p / T::H, h = p % T::H;
        const char *const at_a = smem + buf * T::STAGE, *const at_b = at_a + T::PL * T::PLANE_A;
#pragma unroll
        for (int q = 0; q < T::PL; ++q) {
            if constexpr (h == 0) {
#pragma unroll
                for (int i = 0; i < T::FN; ++i) bv[s][q][i] = b.fragment(at_b + q * T::PLANE_B, wn * T::FN + i, s);
            }
#pragma unroll
            for (int j = 0; j < T::HB; ++j) av[p & 1][q][j] = a.fragment(at_a + q * T::PLANE_A, wt * T::FT + h * T::HB + j, s);
        }
    };
    auto products = [&](auto phase) {
        constexpr int p = decltype(phase)::value, s = p / T::H, h = p % T::H;
#pragma unroll
        for (int t = T::PL == 2 ? 0 : 2; t < 3; ++t)
#pragma unroll
            for (int j = 0; j < T::HB; ++j)
#pragma unroll
                for (int i = 0; i < T::FN; ++i) {
                    f32x4& sum = (APART && t < 2) || (HALVES && s == 1) ? apart[HALVES && t == 2 ? 1 : 0][APART ? i : 0][APART ? h * T::HB + j : 0] : acc[i][h * T::HB + j];
                    sum = multiply16<DT>(bv[s][t == 1 ? 1 : 0][i], av[p & 1][t == 0 ? 1 : 0][j], sum);
                }
    };
    constexpr int PHASES = 2 * T::H, LOADS = T::PL * (T::LA + T::LW);
    typedef std::integral_constant<int, 0> First;
    typedef std::integral_constant<int, PHASES - 1> Last;

    auto multiply_all = [&]() {
        if constexpr (DIRECT) {
            int ks = ks0;  // the next step to load
            auto load = [&](int buf) {
                char* const to = smem + buf * T::STAGE;
                a.load(to, ks < ks1);
                b.load(to + T::PL * T::PLANE_A, ks < ks1);
                ++ks;
                a.advance(), b.advance();
            };

            // Order of a phase of many products: after every few one of its LDS reads, then one of its loads, so that products begin at
            // once.  With few products the reads come first, or they would be late.
            constexpr bool MIXED = T::HB * T::FN * (2 * T::PL - 1) >= 16;
            constexpr int READS_A = T::PL * T::HB * (A_ACROSS ? 2 : 1), READS_B = T::PL * T::FN * (B_ACROSS ? 2 : 1);
            auto interleave = [&](auto reads, auto loads) {
                constexpr int R = decltype(reads)::value, L = decltype(loads)::value, M = T::HB * T::FN * (2 * T::PL - 1), EACH = MIXED ? M / (R + L) : 1;
                if constexpr (MIXED && EACH > 0) {
                    count_to<R>([&](auto) {
                        __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);  // products
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);     // an LDS read
                    });
                    count_to<L>([&](auto) {
                        __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);
                        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);     // a load
                    });
                    if constexpr (M > EACH * (R + L)) __builtin_amdgcn_sched_group_barrier(0x008, M - EACH * (R + L), 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            auto reads_first = [&]() {
                if constexpr (!MIXED) __builtin_amdgcn_sched_barrier(0);
            };
            // Steps past the last are asked for as well, without a byte in range, so that the count of loads on their way is always the same.
#pragma unroll
            for (int k = 0; k < T::S; ++k) load(k);
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::S - 1) * LOADS) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            fetch(0, First());
            int buf = 0;
            for (int k = 0; k < steps - 1; ++k) {
                count_to<PHASES - 1>([&](auto p) {
                    fetch(buf, std::integral_constant<int, decltype(p)::value + 1>());
                    reads_first();
                    products(p);
                    interleave(std::integral_constant<int, READS_A + ((decltype(p)::value + 1) % T::H == 0 ? READS_B : 0)>(), std::integral_constant<int, 0>());
                });
                // this wave's loads of the next stage have landed and its reads of the present one are done; then so are everybody's
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::S - 2) * LOADS) : "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                const int next = buf + 1 == T::S ? 0 : buf + 1;
                fetch(next, First());
                load(buf);
                reads_first();
                products(Last());
                interleave(std::integral_constant<int, READS_A + READS_B>(), std::integral_constant<int, LOADS>());
                buf = next;
            }
            const int tail = ks1 < g.ksteps ? T::KE : (int)(g.K - (int64_t)(g.ksteps - 1) * T::KE);
            count_to<PHASES>([&](auto p) {
                constexpr int q = decltype(p)::value, s = q / T::H;
                if constexpr (q + 1 < PHASES) fetch(buf, std::integral_constant<int, q + 1>());
                const int left = tail - (s * 4 + (lane >> 4)) * 8;
                if constexpr (q % T::H == 0 && !B_ACROSS) {
#pragma unroll
                    for (int i = 0; i < T::PL * T::FN; ++i) bv[s][i / T::FN][i % T::FN] = first_elems(bv[s][i / T::FN][i % T::FN], left);
                }
                if constexpr (!A_ACROSS) {
#pragma unroll
                    for (int j = 0; j < T::PL * T::HB; ++j) av[q & 1][j / T::HB][j % T::HB] = first_elems(av[q & 1][j / T::HB][j % T::HB], left);
                }
                products(p);
            });
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing may land in LDS after the end
        } else {
            static_assert(DIRECT || (T::S == 2 && T::PL == 1), "one stage is multiplied, the other written");
            constexpr int D = decltype(a)::D;
            static_assert(D % 2 == 0, "step k lies in stage k % 2 and came by slot k % D");
            auto load = [&](auto slot) { a.pieces.load(a.held[decltype(slot)::value]), b.pieces.load(b.held[decltype(slot)::value]); };
            auto load_whole = [&](auto slot) { a.template load_whole<decltype(slot)::value>(), b.template load_whole<decltype(slot)::value>(); };
            auto commit = [&](auto slot, auto whole) {
                constexpr int S = decltype(slot)::value;
                char* const to = smem + S % 2 * T::STAGE;
                a.template commit<S, decltype(whole)::value>(to);
                b.template commit<S, decltype(whole)::value>(to + T::PLANE_A);
            };
            auto multiply = [&](auto slot) {
                constexpr int BUF = decltype(slot)::value % 2;
                fetch(BUF, First());
                count_to<PHASES>([&](auto p) {
                    constexpr int q = decltype(p)::value;
                    if constexpr (q + 1 < PHASES) fetch(BUF, std::integral_constant<int, q + 1>());
                    products(p);
                });
            };
            // Step k is in its stage, steps k + 1 .. k + D on their way.  The first loop's loads are of whole steps, without a branch: behind one that
            // may load or not a wave waits for all that is on its way.
            const int whole = min(steps, min(a.pieces.whole(), b.pieces.whole()));
            int k = 0;
            if (whole > 2 * D) {
                count_to<D>(load_whole);
                commit(First(), std::true_type());
                load_whole(First());
                __syncthreads();
                for (; k + 2 * D < whole; k += D) {
                    count_to<D>([&](auto u) {
                        typedef std::integral_constant<int, (decltype(u)::value + 1) % D> Next;
                        multiply(u);
                        commit(Next(), std::true_type());
                        load_whole(Next());
                        __syncthreads();
                    });
                }
            } else {
                count_to<D>(load);
                commit(First(), std::false_type());
                load(First());
                __syncthreads();
            }
            while (k < steps) {
                count_to<D>([&](auto u) {
                    typedef std::integral_constant<int, (decltype(u)::value + 1) % D> Next;
                    if (k >= steps) return;
                    multiply(u);
                    if (++k < steps) commit(Next(), std::false_type());
                    load(Next());  // (past the last step: nothing)
                    __syncthreads();
                });
            }
        }
    };
    auto scale = [&](float by) {
#pragma unroll
        for (int i = 0; i < T::FN; ++i)
#pragma unroll
            for (int j = 0; j < T::FT; ++j) acc[i][j] *= by;
    };
    if constexpr (PARTS) {
        multiply_all();
        scale(1.0f / Parts<DT>::LOW);
        __syncthreads();  // every wave has read its last operands before others land in their place
        begin(0);
        multiply_all();
        if constexpr (Parts<DT>::HIGH != 1.0f) scale(1.0f / Parts<DT>::HIGH);
    } else {
        multiply_all();
    }

    if constexpr (APART) {
#pragma unroll
        for (int i = 0; i < T::FN; ++i)
#pragma unroll
            for (int j = 0; j < T::FT; ++j) {
                if constexpr (HALVES) acc[i][j] += apart[1][i][j];
                acc[i][j] += apart[0][i][j];
            }
    }
    const int grp = lane >> 4;
#pragma unroll
    for (int i = 0; i < T::FN; i += 2) {
        const int nl = (wn * T::FN + i) * 16 + (grp & 1) * 16 + (grp >> 1) * 8;
#pragma unroll
        for (int j = 0; j < T::FT; ++j) {
            const int ml = (wt * T::FT + j) * 16 + (lane & 15);
            float v[8];
            eight_in_a_row(acc[i][j], acc[i + 1][j], v);
            if (ml < a.here && nl < b.here) Epi::finish(g, e, v, g.m_first + m0 + ml, n0 + nl, min(8, b.here - nl), bias + nl);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The sums of workgroups that share a reduction, as they are.
struct PartialSums {
    struct Args {};
    static constexpr bool SYMMETRIC = false;
    static __device__ __forceinline__ void prepare(const Args&, float*, int64_t, int, int, int) {}
    static __device__ __forceinline__ void finish(const ProductArgs& g, const Args&, const float (&v)[8], int64_t m, int64_t n, int have, const float*)
    {
        put8<CONV_F32>(g.partial, ((int64_t)(blockIdx.x % g.splits) * g.M + m) * g.N + n, v, have);
    }
};

}  // namespace convfwd
