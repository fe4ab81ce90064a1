// Matrix product in 8-bit integers with scales for each row and output channel.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <type_traits>

#include "rows_common.h"

namespace convfwd {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;

// Added to an offset within a tile (below 2^31), puts it past the end of any descriptor here.
constexpr uint32_t kFar = 0x80000000u;

// The first `n` bytes of a 16-byte piece (n may be <= 0 or >= 16), the others zero.
__device__ __forceinline__ i32x4 first_bytes(i32x4 v, int n)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int have = n - 4 * i;
        v[i] = have >= 4 ? v[i] : have <= 0 ? 0 : (int)((uint32_t)v[i] & ((1u << (8 * (have & 3))) - 1u));
    }
    return v;
}

__device__ __forceinline__ float finish(int acc, float scale, float bias, int relu)
{
    const float v = (float)acc * scale + bias;
    return relu && v < 0.0f ? 0.0f : v;  // a NaN stays
}

template <int N, typename F>
__device__ __forceinline__ void for_each(F f)
{
    if constexpr (N > 0) {
        for_each<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

// Any strides: a wave 16 channels x 16 rows, operands from memory straight into registers.
template <int DT>
__global__ __launch_bounds__(256) void int_linear_any(IntLinearArgs g)
{
    typedef typename Prec<DT>::elem_t elem_t;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = (blockIdx.x * 4 + wave) * 16;
    const int64_t t0 = (int64_t)blockIdx.y * 16;
    if (n0 >= g.N) return;
    const int i = lane & 15, kq = (lane >> 4) * 16;
    const int8_t* w = g.w + (int64_t)min(n0 + i, g.N - 1) * g.ldw;
    const int8_t* a = g.a + min(t0 + i, g.rows - 1) * g.lda;
    i32x4 acc = {0, 0, 0, 0};
    for (int k = kq; k - kq < g.K; k += 64) {
        i32x4 wv = {0, 0, 0, 0}, av = wv;
        if (k < g.K) {
            wv = first_bytes(*(const i32x4*)(w + k), g.K - k);
            av = *(const i32x4*)(a + k);
        }
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, av, acc, 0, 0, 0);
    }
    const int64_t t = t0 + i;
    if (t >= g.rows) return;
    const float sa = g.a_scale[t];
    elem_t* out = (elem_t*)g.out + t * g.ldo;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int n = n0 + (lane >> 4) * 4 + r;
        if (n < g.N) out[n] = Prec<DT>::from_f32(finish(acc[r], sa * g.w_scale[n], g.bias ? g.bias[n] : 0.0f, g.relu));
    }
}

// Few rows: a workgroup 16 channels x 16 RB rows, its W waves share the reduction: wave w takes every W-th run of 64 U bytes.  The
// weights' stream is what counts, so loads are made of four lanes a 64-byte stretch of a row (a lane a row, as the matrix
// instruction wants them, is served 16 bytes a clock: 64 x 100 x 16384 took 20 us instead of 12), straight into LDS the wave has for
// itself, no barrier; a row's four pieces lie at piece ^ (row / 4 % 4) there, so that no two of 16 lanes read a bank.  The
// waves' exact sums meet in LDS.  Where there are few workgroups and a long reduction, gridDim.z of them share it (int_linear_join).
template <int DT, int RB, int W, int U>
__global__ __launch_bounds__(64 * W) void int_linear_rows(IntLinearArgs g)
{
    typedef typename Prec<DT>::elem_t elem_t;
    constexpr int NT = 64 * W, RUN = 64 * U, OWN = (1 + RB) * U * 1024;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16;
    const int64_t t0 = (int64_t)blockIdx.y * (16 * RB);
    const int Kr = (g.K + 15) & ~15;
    const int rows_here = (int)min((int64_t)(16 * RB), g.rows - t0), outs_here = min(16, g.N - n0);
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(g.a + t0 * g.lda, (uint32_t)((rows_here - 1) * g.lda + Kr));
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(g.w + (int64_t)n0 * g.ldw, (uint32_t)((outs_here - 1) * g.ldw + Kr));
    const int row = lane >> 2, piece = (lane & 3) ^ ((row >> 2) & 3);
    const uint32_t woff = (uint32_t)row * (uint32_t)g.ldw + piece * 16, aoff = (uint32_t)row * (uint32_t)g.lda + piece * 16;
    char* const own = smem + wave * OWN;
    const char* const mine = own + (lane & 15) * 64 + (((lane >> 4) ^ ((lane >> 2) & 3)) << 4);

    i32x4 acc[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) acc[j] = i32x4{0, 0, 0, 0};
    for (int k = (blockIdx.z * W + wave) * RUN; k < g.K; k += gridDim.z * W * RUN) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_void*)(own + u * 1024), 16, (int)(woff + k + u * 64), 0, 0, 0);
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int u = 0; u < U; ++u)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(own + ((1 + j) * U + u) * 1024), 16,
                                                         (int)(aoff + (uint32_t)(j * 16) * (uint32_t)g.lda + k + u * 64), 0, 0, 0);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        i32x4 wv[U], av[RB][U];
#pragma unroll
        for (int u = 0; u < U; ++u) wv[u] = *(const i32x4*)(mine + u * 1024);
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int u = 0; u < U; ++u) av[j][u] = *(const i32x4*)(mine + ((1 + j) * U + u) * 1024);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next run's loads may land
        if (k + RUN > g.K) {
#pragma unroll
            for (int u = 0; u < U; ++u) wv[u] = first_bytes(wv[u], g.K - k - u * 64 - (lane >> 4) * 16);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < RB; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u], av[j][u], acc[j], 0, 0, 0);
    }
    __syncthreads();
    i32x4* const part = (i32x4*)smem;
#pragma unroll
    for (int j = 0; j < RB; ++j) part[(wave * RB + j) * 64 + lane] = acc[j];
    __syncthreads();
    for (int o = threadIdx.x; o < 256 * RB; o += NT) {
        const int n = n0 + (o & 15), r = o >> 4;  // channel; row among the workgroup's
        if (n >= g.N || r >= rows_here) continue;
        int sum = 0;
#pragma unroll
        for (int v = 0; v < W; ++v) sum += ((const int*)&part[(v * RB + (r >> 4)) * 64 + ((o & 15) >> 2) * 16 + (r & 15)])[o & 3];
        if (gridDim.z > 1)
            g.ws[(blockIdx.z * g.rows + t0 + r) * g.N + n] = sum;
        else
            ((elem_t*)g.out)[(t0 + r) * g.ldo + n] =
                Prec<DT>::from_f32(finish(sum, g.a_scale[t0 + r] * g.w_scale[n], g.bias ? g.bias[n] : 0.0f, g.relu));
    }
}

// Adds the sums of `splits` workgroups that shared a reduction.
template <int DT>
__global__ __launch_bounds__(256) void int_linear_join(IntLinearArgs g, int splits)
{
    const int64_t o = (int64_t)blockIdx.x * 256 + threadIdx.x, all = g.rows * g.N;
    if (o >= all) return;
    const int64_t t = o / g.N;
    const int n = (int)(o - t * g.N);
    int sum = 0;
    for (int z = 0; z < splits; ++z) sum += g.ws[z * all + o];
    ((typename Prec<DT>::elem_t*)g.out)[t * g.ldo + n] =
        Prec<DT>::from_f32(finish(sum, g.a_scale[t] * g.w_scale[n], g.bias ? g.bias[n] : 0.0f, g.relu));
}

// Tiles of BT rows x BN channels, both operands staged through LDS by loads that write it directly, a ring of S stages of 128 bytes
// of each row: while one is multiplied, S - 1 are on their way or there.
//   * A row's eight 16-byte pieces are stored at piece ^ (row / 2 % 8), by choosing which piece a lane loads: the 16 lanes that LDS
//     serves together then read 16 different groups of four banks (no conflict counted).
//   * LATE, for rows that begin inside a line of 128 bytes: the 128 bytes of a step would lie in two lines, and every line be asked
//     for twice.  A row's load of step k is the line that its bytes of step k begin in; the pieces behind them come with the load of
//     step k + 1, so a step reads two stages of the ring, each lane its pieces of the one or the other.
//   * Rows past the last one, and pieces past the end of the tensor, are read as zeros by the bounds check of the buffer
//     descriptor; the bytes of a row past K belong to what follows and are cleared in one operand on the last step.
//   * Products are 16x16x64: on random operands the register-only loop reaches 3970 TOP/s with two waves a SIMD, 32x32x32 3480
//     (on zeros both 4600: the card's power sets the clock).
template <int WT_, int WN_, int FT_, int FN_, int S_, bool LATE_>
struct IntTile {
    static constexpr int WT = WT_, WN = WN_, FT = FT_, FN = FN_;  // waves and 16-wide blocks a wave, along rows and channels
    static constexpr int BT = 16 * WT * FT, BN = 16 * WN * FN, NT = 64 * WT * WN;
    static constexpr int KB = 128, S = S_, PIECES = KB / 16;
    static constexpr bool LATE = LATE_;
    static_assert(S >= 2 + LATE, "a stage to multiply, one to load");
    static constexpr int STAGE = (BT + BN) * KB;
    static constexpr int PITCH = BN * 2 + 16;  // of a row of 16-bit outputs in LDS
    static constexpr int RING = S * STAGE > BT * PITCH ? S * STAGE : BT * PITCH;
    static constexpr size_t LDS = (size_t)RING + (BT + 2 * BN) * 4;
    static constexpr int LA = BT * PIECES / NT, LW = BN * PIECES / NT;  // 16-byte loads a thread and stage
    static constexpr int H = FT > 4 ? 2 : 1, HB = FT / H;               // the blocks of rows go in H portions
    static_assert(LA * NT == BT * PIECES && LW * NT == BN * PIECES && FN % 2 == 0 && HB * H == FT, "whole loads and portions");
};

template <int DT, typename T>
__global__ __launch_bounds__(T::NT) void int_linear_tiles(IntLinearArgs g, int tiles_t, int tiles_n)
{
    typedef typename Prec<DT>::elem_t elem_t;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wt = wave % T::WT, wn = wave / T::WT;

    // consecutive workgroups go to different XCDs: each XCD takes a run of tiles, in bands of eight tiles of channels
    const int total = tiles_t * tiles_n;
    int tile = blockIdx.x;
    {
        const int q = total / 8, r = total % 8, x = tile % 8, i = tile / 8;
        tile = x * q + min(x, r) + i;
    }
    const int band = tile / (8 * tiles_t), in_band = tile - band * 8 * tiles_t;
    const int width = min(8, tiles_n - band * 8);
    const int tn = band * 8 + in_band % width, tt = in_band / width;
    const int64_t t0 = (int64_t)tt * T::BT;
    const int n0 = tn * T::BN;

    const int Kr = (g.K + 15) & ~15;
    const int rows_here = (int)min((int64_t)T::BT, g.rows - t0), outs_here = min(T::BN, g.N - n0);
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(g.a + t0 * g.lda, (uint32_t)((rows_here - 1) * g.lda + Kr));
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(g.w + (int64_t)n0 * g.ldw, (uint32_t)((outs_here - 1) * g.ldw + Kr));
    uint32_t aoff[T::LA], woff[T::LW];
    bool alate[T::LA], wlate[T::LW];
    constexpr int P = T::PIECES;
    // the distance of a row's start to the last multiple of 128 bytes, in pieces; the same in rows 16 apart
    auto shift = [](const int8_t* p, int64_t ld, int row) { return T::LATE ? (int)(((uint32_t)((uintptr_t)p >> 4) + row * (uint32_t)(ld >> 4)) % P) : 0; };
#pragma unroll
    for (int i = 0; i < T::LA; ++i) {
        const int p = i * T::NT + tid, row = p / P, piece = (p % P) ^ ((row >> 1) % P);
        alate[i] = piece + shift(g.a, g.lda, row) >= P;
        aoff[i] = (uint32_t)row * (uint32_t)g.lda + (piece << 4) - (alate[i] ? T::KB : 0);
    }
#pragma unroll
    for (int i = 0; i < T::LW; ++i) {
        const int p = i * T::NT + tid, row = p / P, piece = (p % P) ^ ((row >> 1) % P);
        wlate[i] = piece + shift(g.w, g.ldw, row) >= P;
        woff[i] = (uint32_t)row * (uint32_t)g.ldw + (piece << 4) - (wlate[i] ? T::KB : 0);
    }
    const int steps = (g.K + T::KB - 1) / T::KB;
    // Steps past the last are asked for as well, out of range, so that the count of loads on their way is always the same.
    auto stage = [&](int buf, int k, auto first) {
        const uint32_t k0 = k < steps + T::LATE ? (uint32_t)k * T::KB : kFar;
        char* base = smem + buf * T::STAGE + wave * 1024;
#pragma unroll
        for (int i = 0; i < T::LA; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(base + i * T::NT * 16), 16, (int)(first() && alate[i] ? kFar : aoff[i] + k0), 0, 0, 0);
#pragma unroll
        for (int i = 0; i < T::LW; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_void*)(base + T::BT * T::KB + i * T::NT * 16), 16, (int)(first() && wlate[i] ? kFar : woff[i] + k0), 0, 0, 0);
    };

    // the tile's scales and biases wait in LDS for the end
    float* const sc_a = (float*)(smem + T::RING);
    float* const sc_w = sc_a + T::BT;
    float* const bias = sc_w + T::BN;
    for (int i = tid; i < T::BT; i += T::NT) sc_a[i] = i < rows_here ? g.a_scale[t0 + i] : 0.0f;
    for (int i = tid; i < T::BN; i += T::NT) {
        sc_w[i] = i < outs_here ? g.w_scale[n0 + i] : 0.0f;
        bias[i] = g.bias && i < outs_here ? g.bias[n0 + i] : 0.0f;
    }

    int frag[2];  // LDS offset of this lane's piece for each half of a stage, without the block
#pragma unroll
    for (int s = 0; s < 2; ++s) frag[s] = (lane & 15) * T::KB + (((s * 4 + (lane >> 4)) ^ ((lane >> 1) & 7)) << 4);
    // whether that piece is one of the next stage
    bool a_next[2], w_next[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        a_next[s] = s * 4 + (lane >> 4) + shift(g.a, g.lda, lane & 15) >= P;
        w_next[s] = s * 4 + (lane >> 4) + shift(g.w, g.ldw, lane & 15) >= P;
    }
    const int wave_a = wt * T::FT * 16 * T::KB, wave_w = (T::BT + wn * T::FN * 16) * T::KB;

    i32x4 acc[T::FN][T::FT];
#pragma unroll
    for (int i = 0; i < T::FN; ++i)
#pragma unroll
        for (int j = 0; j < T::FT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};

    i32x4 av[2][T::HB], wv[2][T::FN];
    // The operands of phase p of a stage (half p / H, portion p % H of the rows) to the registers of its parity.
    auto fetch = [&](int buf, auto phase) {
        constexpr int p = decltype(phase)::value, s = p / T::H, h = p % T::H;
        const int here = buf * T::STAGE + frag[s], there = buf + 1 == T::S ? frag[s] : here + T::STAGE;
        const char *base = smem + (T::LATE && a_next[s] ? there : here), *base_w = smem + (T::LATE && w_next[s] ? there : here);
        if constexpr (h == 0) {
#pragma unroll
            for (int i = 0; i < T::FN; ++i) wv[s][i] = *(const i32x4*)(base_w + wave_w + i * 16 * T::KB);
        }
#pragma unroll
        for (int j = 0; j < T::HB; ++j) av[p & 1][j] = *(const i32x4*)(base + wave_a + (h * T::HB + j) * 16 * T::KB);
    };
    auto products = [&](auto phase) {
        constexpr int p = decltype(phase)::value, s = p / T::H, h = p % T::H;
#pragma unroll
        for (int j = 0; j < T::HB; ++j)
#pragma unroll
            for (int i = 0; i < T::FN; ++i)
                acc[i][h * T::HB + j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[s][i], av[p & 1][j], acc[i][h * T::HB + j], 0, 0, 0);
    };
    constexpr int PHASES = 2 * T::H, LOADS = T::LA + T::LW;
    typedef std::integral_constant<int, 0> First;
    typedef std::integral_constant<int, PHASES - 1> Last;
    typedef std::integral_constant<int, 0> Zero;
    // Order of a phase of many products: after every few one of its LDS reads, then one of its loads, so that products begin at once
    // (256 x 256: 229 -> 225 us at 8192 x 8192 x 4096).  With few products the reads come first, or they would be late (64 x 64: 10.1 -> 9.5).
    constexpr bool MIXED = T::HB * T::FN >= 16;
    auto interleave = [&](auto reads, auto loads) {
        constexpr int R = decltype(reads)::value, L = decltype(loads)::value, M = T::HB * T::FN, EACH = MIXED ? M / (R + L) : 1;
        if constexpr (MIXED) {
            for_each<R>([&](auto) {
                __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0);  // products
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);     // an LDS read
            });
            for_each<L>([&](auto) {
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
    // Operands are read one phase ahead of their products, across the turn to the next stage too; left to itself the compiler reads
    // them where they are used.
#pragma unroll
    for (int k = 0; k < T::S; ++k) k == 0 ? stage(k, k, std::bool_constant<T::LATE>()) : stage(k, k, std::false_type());
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::S - 1 - T::LATE) * LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    fetch(0, First());
    int buf = 0;
    for (int k = 0; k < steps - 1; ++k) {
        for_each<PHASES - 1>([&](auto p) {
            fetch(buf, std::integral_constant<int, decltype(p)::value + 1>());
            reads_first();
            products(p);
            interleave(std::integral_constant<int, T::HB + ((decltype(p)::value + 1) % T::H == 0 ? T::FN : 0)>(), Zero());
        });
        // this wave's loads of the next stage have landed and its reads of the present one are done; then so are everybody's
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((T::S - 2 - T::LATE) * LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const int next = buf + 1 == T::S ? 0 : buf + 1;
        fetch(next, First());
        stage(buf, k + T::S, std::false_type());
        reads_first();
        products(Last());
        interleave(std::integral_constant<int, T::HB + T::FN>(), std::integral_constant<int, LOADS>());
        buf = next;
    }
    for_each<PHASES>([&](auto p) {
        constexpr int q = decltype(p)::value;
        if constexpr (q + 1 < PHASES) fetch(buf, std::integral_constant<int, q + 1>());
        if constexpr (q % T::H == 0) {
#pragma unroll
            for (int i = 0; i < T::FN; ++i)
                wv[q / T::H][i] = first_bytes(wv[q / T::H][i], g.K - (steps - 1) * T::KB - (q / T::H * 4 + (lane >> 4)) * 16);
        }
        products(p);
    });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing may land in LDS after the end

    // A lane has four channels 4 (lane / 16) .. of a block and row lane % 16 of a block of rows.  In 16 bits neighbouring groups of 16
    // lanes trade between two blocks of channels, so that a lane has eight channels in a row: the groups 0 .. 3 those of block i from
    // 0, of block i + 1 from 0, of block i from 8, of block i + 1 from 8.
    const int grp = lane >> 4;
    // An odd row length puts every other row's elements across words, and a store of half a word is slow: such tiles are turned in LDS and
    // leave in aligned pieces of 16 bytes (4096 x 11009 x 512 71 -> 52 us, 8192 x 50257 x 768 600 -> 567, against stores as they come).
    const bool staged = DT != CONV_F32 && ((g.ldo | (int64_t)((uintptr_t)g.out >> 1)) & 1);
    if (staged) __syncthreads();
#pragma unroll
    for (int i = 0; i < T::FN; i += 2) {
        const int nl = (wn * T::FN + i) * 16;
        float sw[8], b[8];
        __builtin_memcpy(sw, sc_w + nl + grp * 4, 16);
        __builtin_memcpy(sw + 4, sc_w + nl + 16 + grp * 4, 16);
        __builtin_memcpy(b, bias + nl + grp * 4, 16);
        __builtin_memcpy(b + 4, bias + nl + 16 + grp * 4, 16);
#pragma unroll
        for (int j = 0; j < T::FT; ++j) {
            const int tl = (wt * T::FT + j) * 16 + (lane & 15);
            const float sa = sc_a[tl];
            const bool in = tl < rows_here;
            elem_t* out = (elem_t*)g.out + (t0 + tl) * g.ldo + n0;
            float v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = finish(acc[i + (r >> 2)][j][r & 3], sa * sw[r], b[r], 0);
            if (g.relu) {
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = v[r] < 0.0f ? 0.0f : v[r];
            }
            constexpr int LEN = 16 / sizeof(elem_t);
            uint32_t w4[8 / LEN][4];
            int n[8 / LEN];
            if constexpr (DT == CONV_F32) {
                __builtin_memcpy(w4, v, 32);
                n[0] = nl + grp * 4, n[1] = nl + 16 + grp * 4;
            } else {
                const auto r0 = __builtin_amdgcn_permlane16_swap(Prec<DT>::pack2_from_f32(v[0], v[1]), Prec<DT>::pack2_from_f32(v[4], v[5]), false, false);
                const auto r1 = __builtin_amdgcn_permlane16_swap(Prec<DT>::pack2_from_f32(v[2], v[3]), Prec<DT>::pack2_from_f32(v[6], v[7]), false, false);
                w4[0][0] = r0[0], w4[0][1] = r1[0], w4[0][2] = r0[1], w4[0][3] = r1[1];
                n[0] = nl + (grp & 1) * 16 + (grp >> 1) * 8;
            }
#pragma unroll
            for (int c = 0; c < 8 / LEN; ++c) {
                if (staged) {
                    __builtin_memcpy(smem + tl * T::PITCH + n[c] * 2, w4[c], 16);
                } else if (in && n[c] + LEN <= outs_here) {
                    __builtin_memcpy(out + n[c], w4[c], 16);
                } else if (in) {
                    elem_t e[LEN];
                    __builtin_memcpy(e, w4[c], 16);
#pragma unroll
                    for (int r = 0; r < LEN; ++r)
                        if (n[c] + r < outs_here) out[n[c] + r] = e[r];
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (DT != CONV_F32) {
        if (!staged) return;
        __syncthreads();
        constexpr int EACH = T::BN / 8 + 1;  // aligned pieces that a row of the tile touches
        for (int i = tid; i < T::BT * EACH; i += T::NT) {
            const int tl = i / EACH, piece = i - tl * EACH;
            if (tl >= rows_here) break;
            elem_t* out = (elem_t*)g.out + (t0 + tl) * g.ldo + n0;
            const int e0 = piece * 8 - (int)((uintptr_t)out / 2 % 8);
            if (e0 >= 0 && e0 + 8 <= outs_here) {
                const uint32_t* from = (const uint32_t*)(smem + tl * T::PITCH + (e0 & ~1) * 2);
                uint32_t w[5];
#pragma unroll
                for (int k = 0; k < 5; ++k) w[k] = from[k];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = e0 & 1 ? __builtin_amdgcn_alignbyte(w[k + 1], w[k], 2) : w[k];
                *(uint4*)(out + e0) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        // the pieces that a row's tile shares with its neighbours, an element a lane
        for (int i = tid; i < T::BT * 16; i += T::NT) {
            const int tl = i / 16, half = i / 8 % 2;
            if (tl >= rows_here) break;
            elem_t* out = (elem_t*)g.out + (t0 + tl) * g.ldo + n0;
            const int at = (int)((uintptr_t)out / 2 % 8), last = (outs_here + at) / 8;  // the piece that ends behind the tile
            const int e = (half ? last * 8 : 0) - at + i % 8;
            if (half ? e >= 0 && e < outs_here : at && last && e >= 0) out[e] = *(const elem_t*)(smem + tl * T::PITCH + e * 2);
        }
    }
}

template <int DT, typename T>
hipError_t launch_tiles(const IntLinearArgs& g, hipStream_t s)
{
    const void* f = (const void*)int_linear_tiles<DT, T>;
    const hipError_t e = ensure_dynamic_lds(f, T::LDS);
    if (e != hipSuccess) return e;
    const int tn = (g.N + T::BN - 1) / T::BN;
    // a launch holds less than 2^32 threads: the rows go in portions of so many bands
    const int64_t bands = std::max<int64_t>(1, (1 << 21) / tn);
    for (int64_t skip = 0; skip < g.rows; skip += bands * T::BT) {
        IntLinearArgs p = g;
        p.rows = std::min(bands * T::BT, g.rows - skip);
        p.a += skip * g.lda, p.a_scale += skip, p.out = (char*)g.out + skip * g.ldo * dtype_size(DT);
        const int tt = (int)((p.rows + T::BT - 1) / T::BT);
        hipLaunchKernelGGL((int_linear_tiles<DT, T>), dim3((unsigned)tt * (unsigned)tn), dim3(T::NT), T::LDS, s, p, tt, tn);
    }
    return hipGetLastError();
}

// gridDim.y is at most 65535: the rows go in portions of that many workgroups.
template <int DT, typename F>
hipError_t in_portions(const IntLinearArgs& g, int rows_each, F launch)
{
    const int64_t portion = 65535 * (int64_t)rows_each;
    for (int64_t skip = 0; skip < g.rows; skip += portion) {
        IntLinearArgs p = g;
        p.rows = std::min(portion, g.rows - skip);
        p.a += skip * g.lda, p.a_scale += skip, p.out = (char*)g.out + skip * g.ldo * dtype_size(DT);
        const hipError_t e = launch(p, (unsigned)((p.rows + rows_each - 1) / rows_each));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Tiles, and what a launch of them is expected to take, in us: `once` and for every round of 256 tiles `own` and `step` for every 128
// bytes of the reduction.  The figures were fitted to calls of 134 sizes, 10 to 50257 channels, rows of 32 to 16384 bytes aligned
// and not, each in every form (8-bit codes at random, bf16 out): what the rule below takes was 1.8 % slower than the best form on
// average, 20 % at most.  LATE: see IntTile; 64x64 at 256 x 13632 x 16287 193 -> 147 us, 128x128 121 -> 96, 256x256 has no room for
// a third stage.
template <bool LATE> using Tile64x64 = IntTile<4, 2, 1, 2, 4, LATE>;
template <bool LATE> using Tile64x128 = IntTile<2, 4, 2, 2, LATE ? 4 : 3, LATE>;
template <bool LATE> using Tile128x128 = IntTile<4, 4, 2, 2, 4, LATE>;
typedef IntTile<2, 4, 4, 2, 2, false> Pair128x128;  // two workgroups a CU: one stores its tile while the other multiplies
typedef IntTile<4, 2, 4, 8, 2, false> Tile256x256;
// Measured (us of the GPU, bf16 out), rows / 64x64 / 64x128 / 128x128 / two 128x128 a CU / 256x256:
//   512 x 4096 x 4096 37 / 19 / 16 / 19 / 23 / 42;  1024 x 4096 x 1024 22 / 12 / 15 / 9.7 / 9.4 / 17;  2048 x 2048 x 2048 38 / 19 / 16 / 17 / 16 / 26;
//   5298 x 608 x 5120 79 / 36 / 28 / 25 / 33 / 56;  8192 x 1024 x 4096 123 / 61 / 46 / 44 / 38 / 46;  4096 x 4096 x 4096 263 / 114 / 90 / 85 / 71 / 57;
//   8192 x 50256 x 768 1780 / 816 / 611 / 618 / 489 / 526;  8192 x 8192 x 64 161 / 87 / 57 / 60 / 41 / 38;
//   8192 x 8192 x 4096 1030 / 443 / 371 / 345 / 304 / 242 (in later runs 217 to 221, 2500 TOP/s, and 3300 on zeros: the card's power holds
//   the clock down.  The register-only loop has 3970 and 4600: what is missing on zeros too is no power but the ring of two stages, which
//   waits for all its loads at every step with no other workgroup on the CU; waves wait for 32 % of their cycles.)
template <typename T>
double tiles_us(const IntLinearArgs& g, double once, double own, double step)
{
    const double tiles = (double)((g.rows + T::BT - 1) / T::BT) * ((g.N + T::BN - 1) / T::BN), steps = (g.K + T::KB - 1) / T::KB;
    return once + std::ceil(tiles / 256) * (own + steps * step);
}

// Few rows: blocks of 16 rows a workgroup, workgroups that share a reduction, expected us.  A workgroup reads 120 KB in a us, all of
// them 33 TB/s (from the caches mostly), and one takes 0.16 us of a CU a block at least; a second launch to add shares costs about 5 us of a
// call, so it has to save more (64 x 100 x 16384 11.9 -> 9.2, but 128 x 128 x 8192 7.8 -> 8.1).
struct RowsPlan {
    int rb, splits;
    double us;
};
RowsPlan rows_plan(int64_t rows, int N, int K)
{
    RowsPlan p;
    p.rb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const double groups = (double)((rows + 16 * p.rb - 1) / (16 * p.rb)) * ((N + 15) / 16);
    const double bytes = 16.0 * (1 + p.rb) * K, alone = bytes / 120e3 * std::ceil(groups / 256);
    p.splits = 1;
    p.us = 2.8 + alone + std::max(groups * bytes / 33e6, groups / 256 * 0.16 * p.rb);
    if (groups <= 64) {
        const int most = std::min({16, (int)(256 / groups), (K + 1023) / 1024});
        if (alone - alone / most > 6) p.splits = most, p.us = 8 + alone / most;
    }
    return p;
}

template <int DT, int RB, int W, int U>
hipError_t launch_rows(const IntLinearArgs& g, int splits, hipStream_t s)
{
    constexpr size_t LDS = (size_t)W * (1 + RB) * U * 1024;
    const hipError_t e = ensure_dynamic_lds((const void*)int_linear_rows<DT, RB, W, U>, LDS);
    if (e != hipSuccess) return e;
    return in_portions<DT>(g, 16 * RB, [&](const IntLinearArgs& p, unsigned y) {
        hipLaunchKernelGGL((int_linear_rows<DT, RB, W, U>), dim3((unsigned)((g.N + 15) / 16), y, (unsigned)splits), dim3(64 * W), LDS, s, p);
        if (splits > 1) hipLaunchKernelGGL((int_linear_join<DT>), dim3((unsigned)((p.rows * p.N + 255) / 256)), dim3(256), 0, s, p, splits);
        return hipGetLastError();
    });
}

// Waves a workgroup: a wave has a run of 256 bytes or more up to 1024 and 2048 bytes; 16 waves were no better
// (us with 4 / 8 / 16: 1 x 4096 x 4096 5.5 / 5.0 / 5.1, 20 x 1000 x 4096 4.5 / 3.7 / 4.0, 16 x 10000 x 1000 4.2 / 5.0 / 6.9).
template <int DT, int RB>
hipError_t launch_rows(const IntLinearArgs& g, int splits, hipStream_t s)
{
    constexpr int U = RB == 1 ? 4 : 2;
    return g.K <= 1024 ? launch_rows<DT, RB, 4, U>(g, splits, s) : launch_rows<DT, RB, 8, U>(g, splits, s);
}

// The tiles' offsets are 32 bits; longer strides go to int_linear_any.
bool long_strides(int64_t lda, int64_t ldw) { return std::max(lda, ldw) >= (1 << 23); }

// The form of a call.
enum FormId { ANY, ROWS16, ROWS32, ROWS64, T64X64, T64X128, T128X128, PAIR128X128, T256X256 };
struct IntForm {
    FormId id;
    int splits;  // of the few-row forms
    bool late;   // of the first three tiles
};
IntForm form_of(const IntLinearArgs& g)
{
    if (long_strides(g.lda, g.ldw)) return {ANY, 1, false};
    const RowsPlan rows = rows_plan(g.rows, g.N, g.K);
    const IntForm few = {rows.rb == 1 ? ROWS16 : rows.rb == 2 ? ROWS32 : ROWS64, rows.splits, false};
    if (rows.rb == 1) return few;
    const bool late = (g.lda | g.ldw | (int64_t)(uintptr_t)g.a | (int64_t)(uintptr_t)g.w) % 128 != 0;
    const bool alone = (g.rows + 127) / 128 * ((g.N + 127) / 128) <= 256;
    const double us[] = {rows.us, tiles_us<Tile64x64<false>>(g, 2.0, 1.2, 0.2), tiles_us<Tile64x128<false>>(g, 1.5, 2.8, 0.33),
                         alone ? tiles_us<Tile128x128<false>>(g, 0, 4.2, 0.49) : tiles_us<Pair128x128>(g, 1.8, 1.5, 0.52),
                         tiles_us<Tile256x256>(g, 0, 11, 1.4)};
    switch ((int)(std::min_element(us, us + 5) - us)) {
        case 0: return few;
        case 1: return {T64X64, 1, late};
        case 2: return {T64X128, 1, late};
        case 3: return alone ? IntForm{T128X128, 1, late} : IntForm{PAIR128X128, 1, false};
        default: return {T256X256, 1, false};
    }
}

template <int DT>
hipError_t launch(IntLinearArgs& g, hipStream_t s)
{
    const IntForm f = form_of(g);
    switch (f.id) {
        case ANY:
            return in_portions<DT>(g, 16, [&](const IntLinearArgs& p, unsigned y) {
                hipLaunchKernelGGL((int_linear_any<DT>), dim3((unsigned)((g.N + 63) / 64), y), dim3(256), 0, s, p);
                return hipGetLastError();
            });
        case ROWS16: return launch_rows<DT, 1>(g, f.splits, s);
        case ROWS32: return launch_rows<DT, 2>(g, f.splits, s);
        case ROWS64: return launch_rows<DT, 4>(g, f.splits, s);
        case T64X64: return f.late ? launch_tiles<DT, Tile64x64<true>>(g, s) : launch_tiles<DT, Tile64x64<false>>(g, s);
        case T64X128: return f.late ? launch_tiles<DT, Tile64x128<true>>(g, s) : launch_tiles<DT, Tile64x128<false>>(g, s);
        case T128X128: return f.late ? launch_tiles<DT, Tile128x128<true>>(g, s) : launch_tiles<DT, Tile128x128<false>>(g, s);
        case PAIR128X128: return launch_tiles<DT, Pair128x128>(g, s);
        default: return launch_tiles<DT, Tile256x256>(g, s);
    }
}

}  // namespace

// (also where another form or the strides turn out to need none: what a caller keeps depends on the sizes alone)
size_t int_linear_workspace(int64_t rows, int N, int K)
{
    if (rows == 0) return 0;
    const RowsPlan p = rows_plan(rows, N, K);
    return p.splits > 1 ? (size_t)p.splits * rows * N * 4 : 0;
}

int int_linear_form_name(const IntLinearArgs& g, char* buf, size_t n)
{
    static const char* const names[] = {"any", "rows16", "rows32", "rows64", "tile64x64", "tile64x128", "tile128x128", "tile128x128_two_a_cu", "tile256x256"};
    const IntForm f = form_of(g);
    if (f.splits > 1) return std::snprintf(buf, n, "%s_split%d", names[f.id], f.splits);
    return std::snprintf(buf, n, "%s%s", names[f.id], f.late ? "_lines" : "");
}

hipError_t launch_int_linear(IntLinearArgs& g, int dtype, hipStream_t s)
{
    return dtype == CONV_F32 ? launch<CONV_F32>(g, s) : dtype == CONV_F16 ? launch<CONV_F16>(g, s) : launch<CONV_BF16>(g, s);
}

}  // namespace convfwd
