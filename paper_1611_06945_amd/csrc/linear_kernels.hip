// Linear layers: out = act(x w^T + bias) + residual, and the gradients.  Which kernels a call takes, the form for few rows, and what stands
// around the products: the gradient of the activation with its column sums, the join of shared reductions.
#include <cstdio>

#include "linear_common.h"

namespace convfwd {

namespace {

// ---- few rows -------------------------------------------------------------------------------------------------------------

struct LinearRows {
    const void *x, *w;
    int64_t ldx, ldw;
    int64_t rows;
    int N, K;
    LinearOut out;
    float* partial;
};

template <int DT>
__device__ __forceinline__ float finish_one(const LinearOut& e, float z, int64_t t, int n)
{
    typedef typename Prec<DT>::elem_t elem_t;
    if (e.bias) z += e.bias[n];
    if (e.pre) ((elem_t*)e.pre)[t * e.ldo + n] = Prec<DT>::from_f32(z);
    float v = act_of<DT>(z, e.act);
    if (e.residual) v += Prec<DT>::to_f32(((const elem_t*)e.residual)[t * e.ldr + n]);
    return v;
}

// One 16-byte piece of 16 rows of either operand, a lane four bytes times four of row lane % 16.  fp32: a lane's four values go to four
// instructions, each of which takes one k of every lane; the order of a sum's terms is free.
template <int DT>
__device__ __forceinline__ f32x4 multiply_pieces(u32x4 w, u32x4 x, f32x4 c)
{
    if constexpr (DT == CONV_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t wk = w[k], xk = x[k];  // (a cast of a vector's element itself takes the first one)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, wk), __builtin_bit_cast(float, xk), c, 0, 0, 0);
        }
        return c;
    } else {
        return multiply16<DT>(w, x, c);
    }
}

// The first `n` elements of a piece (n may be <= 0 or more than it has), the others zero.
template <int DT>
__device__ __forceinline__ u32x4 first_of_piece(u32x4 v, int n)
{
    if constexpr (DT == CONV_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = k < n ? v[k] : 0u;
        return v;
    } else {
        return first_elems(v, n);
    }
}

// A workgroup 16 NB outputs x 16 RB rows, its W waves share the reduction: wave w takes every W-th run of 64 U bytes.  The weights' stream is what
// counts, so loads are made of four lanes a 64-byte stretch of a row (a lane a row, as the matrix instruction wants them, is
// served 16 bytes a clock), straight into LDS the wave has for itself, no barrier; a row's four pieces lie at piece ^ (row / 4 % 4) there, so
// that no two of 16 lanes read a bank.  The waves' sums meet in LDS.  gridDim.z workgroups may share a long reduction (linear_join).
// DIRECT: rows start on 16 bytes; otherwise pieces go through registers.  Bound by the weights' stream: 1 x 4096 x 4096 fp16 7.7 us, 4.4 TB/s from memory
// (a launch, the first loads and the join of waves in it), 1 x 65536 x 4096 bf16 86 us, 6.2 TB/s, in part from the caches.  In fp32 the rows of x, read again for every 16
// outputs, take longer than the weights: NB > 1 where that leaves workgroups for most CUs (24 x 6752 x 46704 320 -> 226 us, 16 x 4099 x 16001 72 -> 54).
template <int DT, int NB, int RB, int W, int U, bool DIRECT>
__global__ __launch_bounds__(64 * W) void linear_rows(LinearRows g)
{
    typedef typename Prec<DT>::elem_t elem_t;
    constexpr int NT = 64 * W, ES = sizeof(elem_t), VEC = 16 / ES, RUN = 64 * U / ES, SLOT = (NB + RB) * U * 1024, OWN = (DIRECT ? 2 : 1) * SLOT;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * (16 * NB);
    const int64_t t0 = (int64_t)blockIdx.y * (16 * RB);
    const int rows_here = (int)min((int64_t)(16 * RB), g.rows - t0), outs_here = min(16 * NB, g.N - n0);
    const elem_t *const x = (const elem_t*)g.x + t0 * g.ldx, *const w = (const elem_t*)g.w + (int64_t)n0 * g.ldw;
    const int row = lane >> 2, piece = (lane & 3) ^ ((row >> 2) & 3);
    char* const own = smem + wave * OWN;
    const int mine = (lane & 15) * 64 + (((lane >> 4) ^ ((lane >> 2) & 3)) << 4);
    // (whole pieces: rows start on 16 bytes, so what the last one holds past the end lies in the same 16 bytes as an element)
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(x, DIRECT ? (uint32_t)(((rows_here - 1) * g.ldx + g.K) * ES + 15) & ~15u : 0u);
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(w, DIRECT ? (uint32_t)(((outs_here - 1) * g.ldw + g.K) * ES + 15) & ~15u : 0u);
    const uint32_t woff = DIRECT ? (uint32_t)row * (uint32_t)(g.ldw * ES) + piece * 16 : 0u;
    const uint32_t xoff = DIRECT ? (uint32_t)row * (uint32_t)(g.ldx * ES) + piece * 16 : 0u;
    // Pieces from any address: all of a run's are asked for, without a branch, before the first is written to LDS.  Lanes without a row read another one's;
    // only the run that holds the reduction's end loads element by element.
    auto pieces = [&](const elem_t* p, int64_t ld, int at, int here, int k, u32x4 (&v)[U]) {
        const elem_t* from = p + (int64_t)min(at, here - 1) * ld + piece * VEC;
        if (k + RUN <= g.K) {
#pragma unroll
            for (int u = 0; u < U; ++u) __builtin_memcpy(&v[u], from + k + u * (64 / ES), 16);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int first = k + u * (64 / ES), n = g.K - first - piece * VEC;
                elem_t e[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) e[j] = j < n ? from[first + j] : (elem_t)0;
                __builtin_memcpy(&v[u], e, 16);
            }
        }
    };

    // (fp32: two sums a wave, of every other 64 bytes, so that a wave's share of a long reduction is no longer chain than the library's)
    constexpr int SUMS = DT == CONV_F32 ? 2 : 1;
    f32x4 acc[SUMS][NB][RB];
#pragma unroll
    for (int a = 0; a < SUMS; ++a)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < RB; ++j) acc[a][i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // DIRECT: a run's loads, into one of two places
    auto ask = [&](int k, char* slot) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_void_t*)(slot + (i * U + u) * 1024), 16,
                                                         (int)(woff + (uint32_t)(i * 16) * (uint32_t)(g.ldw * ES) + (uint32_t)k * ES + u * 64), 0, 0, 0);
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int u = 0; u < U; ++u)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void_t*)(slot + ((NB + j) * U + u) * 1024), 16,
                                                         (int)(xoff + (uint32_t)(j * 16) * (uint32_t)(g.ldx * ES) + (uint32_t)k * ES + u * 64), 0, 0, 0);
    };
    const int first = (blockIdx.z * W + wave) * RUN, step = gridDim.z * W * RUN;
    char* slot = own;
    if (DIRECT && first < g.K) ask(first, slot);
    for (int k = first; k < g.K; k += step) {
        if constexpr (DIRECT) {
            if (k + step < g.K) {
                ask(k + step, slot == own ? own + SLOT : own);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB + RB) * U) : "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
        } else {
            u32x4 got[NB + RB][U];
#pragma unroll
            for (int i = 0; i < NB; ++i) pieces(w, g.ldw, i * 16 + row, outs_here, k, got[i]);
#pragma unroll
            for (int j = 0; j < RB; ++j) pieces(x, g.ldx, j * 16 + row, rows_here, k, got[NB + j]);
#pragma unroll
            for (int j = 0; j < NB + RB; ++j)
#pragma unroll
                for (int u = 0; u < U; ++u) *(u32x4*)(own + (j * U + u) * 1024 + lane * 16) = got[j][u];
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        u32x4 wv[NB][U], xv[RB][U];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int u = 0; u < U; ++u) wv[i][u] = *(const u32x4*)(slot + mine + (i * U + u) * 1024);
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int u = 0; u < U; ++u) xv[j][u] = *(const u32x4*)(slot + mine + ((NB + j) * U + u) * 1024);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next but one run's loads may land
        if (DIRECT) slot = slot == own ? own + SLOT : own;
        if (DIRECT && k + RUN > g.K) {
            // what follows a row's end is another row's, or nobody's
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int n = g.K - k - u * (64 / ES) - (lane >> 4) * VEC;
#pragma unroll
                for (int i = 0; i < NB; ++i) wv[i][u] = first_of_piece<DT>(wv[i][u], n);
#pragma unroll
                for (int j = 0; j < RB; ++j) xv[j][u] = first_of_piece<DT>(xv[j][u], n);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < RB; ++j) acc[u % SUMS][i][j] = multiply_pieces<DT>(wv[i][u], xv[j][u], acc[u % SUMS][i][j]);
    }
    __syncthreads();
    f32x4* const part = (f32x4*)smem;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < RB; ++j) part[((wave * NB + i) * RB + j) * 64 + lane] = SUMS == 2 ? acc[0][i][j] + acc[SUMS - 1][i][j] : acc[0][i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < 256 * NB * RB; o += NT) {
        const int l = o % (16 * NB), n = n0 + l, r = o / (16 * NB);  // output; row among the workgroup's
        if (n >= g.N || r >= rows_here) continue;
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < W; ++v) sum += ((const float*)&part[((v * NB + (l >> 4)) * RB + (r >> 4)) * 64 + ((l & 15) >> 2) * 16 + (r & 15)])[l & 3];
        if (gridDim.z > 1)
            g.partial[((int64_t)blockIdx.z * g.rows + t0 + r) * g.N + n] = sum;
        else
            ((elem_t*)g.out.out)[(t0 + r) * g.out.ldo + n] = Prec<DT>::from_f32(finish_one<DT>(g.out, sum, t0 + r, n));
    }
}

// Adds the sums of `splits` workgroups that shared a reduction, in their order, 16 of them on their way at a time (64 of 768 x 192: 17.5 us one after the
// other, 7.4 so; 4 MB of results of two bytes from 64 MB 15 us).
template <int DT>
__global__ __launch_bounds__(256) void linear_join(LinearOut e, const float* partial, int64_t rows, int N, int splits)
{
    const int64_t o = (int64_t)blockIdx.x * 256 + threadIdx.x, all = rows * N;
    if (o >= all) return;
    const int64_t t = o / N;
    const int n = (int)(o - t * N);
    float sum = 0.0f;
#pragma unroll 16
    for (int z = 0; z < splits; ++z) sum += partial[z * all + o];
    ((typename Prec<DT>::elem_t*)e.out)[t * e.ldo + n] = Prec<DT>::from_f32(finish_one<DT>(e, sum, t, n));
}

// ---- around the products --------------------------------------------------------------------------------------------------

// The gradient at the sum: dz = dout act'(pre), with its sums over the rows.  A workgroup has 256 columns and `each` rows, eight lanes of
// rows; the sums are of the values before they are rounded.
// Bound by memory: 200704 x 768 fp16 with GELU 258 us, 4.8 TB/s of two tensors read and two written.
// TO: whether dz is written, with the row stride ldz: 1 in the storage type, where that holds it (no activation, or ReLU's, whose slopes are 0 and 1); 2 in two
// parts, the low one `plane` elements behind the high one.  (In one part a gradient behind GELU was off by 1.4 times its own rounding, and an fp16 dz could become an infinity or zero.)
template <int DT, int TO>
__global__ __launch_bounds__(256) void linear_dz(const void* dout, const void* pre, int64_t ld, int64_t rows, int N, int act, void* dz, int64_t ldz,
                                                 int64_t plane, float* sums, int64_t each)
{
    __shared__ float lds[8][32 * 8 + 8];
    const int col = threadIdx.x & 31, r = threadIdx.x >> 5;
    const int64_t j = ((int64_t)blockIdx.x * 32 + col) * 8;
    const int have = (int)min((int64_t)8, N - j);
    const int64_t first = blockIdx.y * each, last = min(first + each, rows);
    float sum[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
    if (j < (TO ? ldz : (int64_t)N)) {
        for (int64_t t = first + r; t < last; t += 8) {
            float v[8];
            get8<DT>(dout, t * ld + j, v, have);
            if (act) {
                float z[8];
                get8<DT>(pre, t * ld + j, z, have);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= act_slope(z[k], act);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (k >= have) v[k] = 0.0f;
                sum[k] += v[k];
            }
            const int room = (int)min((int64_t)8, ldz - j);
            if constexpr (TO == 1) put8<DT>(dz, t * ldz + j, v, room);
            if constexpr (TO == 2) {
                float high[8], low[8];
                Parts<DT>::split(v, high, low);
                put8<DT>(dz, t * ldz + j, high, room);
                put8<DT>(dz, plane + t * ldz + j, low, room);
            }
        }
    }
    if (!sums) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) lds[r][k * 33 + col] = sum[k];
    __syncthreads();
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    float all = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) all += lds[i][(threadIdx.x & 7) * 33 + (threadIdx.x >> 3)];
    sums[(int64_t)blockIdx.y * N + n] = all;
}

// Adds `parts` rows of partial sums, always in the same order: a workgroup 32 columns, 32 lanes of rows (341 rows of 768: 13.9 us with eight
// lanes, 4.7 so).
__global__ __launch_bounds__(1024) void linear_sums(const float* part, int parts, int N, float* out)
{
    __shared__ float lds[32][32];
    const int col = threadIdx.x & 31, r = threadIdx.x >> 5, n = blockIdx.x * 32 + col;
    float sum = 0.0f;
    if (n < N) {
#pragma unroll 8
        for (int i = r; i < parts; i += 32) sum += part[(int64_t)i * N + n];
    }
    lds[r][col] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || n >= N) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) sum += lds[i][col];
    out[n] = sum;
}

// What no row adds anything to.
__global__ __launch_bounds__(256) void linear_zero(char* out, int64_t ld_bytes, int64_t rows, int64_t cols_bytes)
{
    const int64_t words = cols_bytes / 2, all = rows * words, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) *(uint16_t*)(out + i / words * ld_bytes + i % words * 2) = 0;
}

// ---- plans ----------------------------------------------------------------------------------------------------------------

constexpr int64_t kLongStride = 1 << 22;  // from here on a tile's offsets may pass 31 bits

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Tiles, and what a launch of them is expected to take, in us: `once` and for every round of 256 tiles `own` and `step` for every 64 of the
// reduction and every part of the first operand.
struct TileCost {
    int bt, bn;
    double once, own, step;
};
constexpr TileCost kTiles[] = {{64, 64, 3.3, 1.1, 0.24}, {128, 128, 2.2, 1.95, 0.51}, {256, 256, 0, 6.6, 1.1}, {192, 192, 0, 5.6, 0.75}, {64, 64, 5.2, 1.7, 0.28}, {128, 128, 2.4, 5.7, 0.59}};
constexpr TileCost kTilesF32[] = {{64, 64, 4.6, 0.75, 1.06}, {128, 128, 0, 6.4, 2.36}, {256, 128, 0, 7.8, 3.9}};

struct ProductPlan {
    ProductForm form;
    int splits;
    double us;
    int64_t rows;      // of the first launch; the rest, if any, by a second one
    ProductForm rest;
    int rest_splits;
};
// across: an operand lies across the reduction, which costs a lone fp32 tile of 64 x 64 more (1024 x 1024 x 1024: 22.5 and 24.3 us; of 128 x 128 in four
// shares 23.7); a CU that has more of these tiles than one has several at a time, whose steps but the first take two thirds of the time (476 of 13 steps 31 us, 1024 of 32 124).
ProductPlan plan_product(int64_t M, int64_t N, int64_t K, int dtype, bool direct, bool across, int parts = 1, bool whole = false)
{
    ProductPlan best = {P64, 1, 1e30, M, P64, 1};
    const int64_t ksteps = (K + 63) / 64;
    const bool f32 = dtype == CONV_F32;
    for (int f = f32 || direct ? P64 : P64_ANY; f <= (f32 ? P256 : direct ? P192 : P128_ANY); ++f) {
        const TileCost& c = f32 ? kTilesF32[f] : kTiles[f];
        const bool small_across = f32 && f == P64 && across;
        const double step = c.step + (small_across ? 0.12 : 0.0), later = small_across ? 0.63 : 1.0;
        const auto time_of = [&](double turns, int64_t steps) { return turns * (c.own + step) + ((1 + later * (turns - 1)) * (parts * steps - 1)) * step; };
        const int64_t tm = (M + c.bt - 1) / c.bt, tn = (N + c.bn - 1) / c.bn;
        const double tiles = (double)tm * tn;
        for (int splits = 1; splits <= 64; splits *= 2) {
            if (splits > 1 && (splits * 4 > ksteps || tiles * splits > 2048)) break;
            const int64_t each = (ksteps + splits - 1) / splits;
            const int shares = (int)((ksteps + each - 1) / each);  // none without a step
            const double turns = std::ceil(tiles * shares / 256);
            double us = c.once + time_of(turns, each);
            if (shares > 1) us += f32 && across ? 4 + 6.0 * shares * M * N / 4e6 : 5 + 8.0 * shares * M * N / 4e6;  // written, read and added by a second launch
            if (us < best.us) best = {(ProductForm)f, shares, us, M, P64, 1};
        }
        // Whole rounds of tiles, and what is left by smaller ones or with a shared reduction (50257 x 1024 x 2048: 788 tiles of 256 x 256 are
        // three rounds and 20 tiles).
        const int64_t rounds = (int64_t)(tiles / 256), first = rounds * 256 / tn;
        if (whole || rounds < 1 || rounds > 16 || first < 1 || first >= tm) continue;
        const ProductPlan rest = plan_product(M - first * c.bt, N, K, dtype, direct, across, parts, true);
        const double us = c.once + time_of(rounds, ksteps) + rest.us;
        if (us < best.us) best = {(ProductForm)f, 1, us, first * c.bt, rest.form, rest.splits};
    }
    return best;
}

// Few rows: blocks of 16 rows a workgroup, workgroups that share a reduction, expected us.  A workgroup reads 120 KB in a us, all of them
// 33 TB/s (from the caches mostly), and one takes 0.16 us of a CU a block at least; a second launch to add shares costs about 5 us of a call.  The fp32 matrix
// instructions, 0.61 MFLOP a us and CU, add half their time: without it 18000 x 576 x 160 took 64 rows a workgroup and 56 us, in tiles 38; 114048 x 576 x 45 122 and 76.
struct RowsPlan {
    int rb, nb, splits;
    double us;
};
// Blocks of 16 outputs a workgroup, in fp32: four, or two of rows that start anywhere, where that makes 192 workgroups or more (20 x 1024 x 8192 in 128 of
// them takes 14 us, one block each 12); 16 rows on 16 bytes take one (57 us for 16 x 4096 x 16000, with two 59), and so do short sums of more than 32 rows (40 x 544 x 45824: 50, with four 53).
int blocks_of_outputs(int64_t rows, int rb, int N, int K, int dtype, bool direct)
{
    const int nb = direct ? 4 : 2;
    if (dtype != CONV_F32 || rows > 64 || K * 4 <= 1024 || N < 192 * 16 * nb) return 1;
    if (rb == 1) return direct ? 1 : nb;
    return rb == 4 && (!direct || K < 1024) ? 1 : nb;
}
RowsPlan plan_rows(int64_t rows, int N, int K, int dtype, bool direct)
{
    RowsPlan p;
    const double size = dtype_size(dtype);
    p.rb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    p.nb = blocks_of_outputs(rows, p.rb, N, K, dtype, direct);
    const double groups = (double)((rows + 16 * p.rb - 1) / (16 * p.rb)) * ((N + 16 * p.nb - 1) / (16 * p.nb));
    const double bytes = 16.0 * (p.nb + p.rb) * K * size, alone = bytes / 120e3 * std::ceil(groups / 256);
    const double matrix = dtype == CONV_F32 ? 0.5 * 2 * 16 * 16 * p.nb * p.rb * (double)K / 0.61e6 : 0.0;
    p.splits = 1;
    // (pieces that start anywhere: twice that for 64 rows, whose loads outweigh the weights')
    p.us = 2.8 + (direct || p.rb < 4 ? 1 : 2) * (alone + std::max(groups * bytes / 33e6, groups / 256 * 0.16 * p.rb)) + matrix * std::ceil(groups / 256);
    if (p.nb > 1) p.us = std::max(p.us, 2.8 + N * (K * size) / 5.3e6 + matrix * std::ceil(groups / 256));  // ... and the weights come from memory
    if (groups <= 64) {
        const int most = std::min({16, (int)(256 / groups), (int)((K * size + 1023) / 1024)});
        if (alone - alone / most > 6) p.splits = most, p.us = 8 + (alone + matrix) / most;
    }
    return p;
}

bool on_16(const void* p, int64_t ld, int size) { return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0 && ld < kLongStride; }

// A forward call: few rows, or tiles.
struct LinearForm {
    bool rows, direct;
    RowsPlan few;
    ProductPlan tiles;
};
LinearForm form_of(int64_t rows, int N, int K, int dtype, bool direct)
{
    LinearForm f;
    f.direct = direct;
    f.few = plan_rows(rows, N, K, dtype, direct);
    f.tiles = plan_product(rows, N, K, dtype, direct, false);
    // (few fp32 rows: tiles take the weights from memory at 3.2 TB/s)
    if (dtype == CONV_F32 && rows <= 64) f.tiles.us = std::max(f.tiles.us, 4 + (double)N * K * 4 / 3.2e6);
    f.rows = rows <= 16 || f.few.us <= f.tiles.us;
    return f;
}

struct Carve {  // pieces of a workspace
    char* at;
    size_t used = 0;
    explicit Carve(void* p) : at((char*)p) {}
    void* take(size_t bytes)
    {
        void* p = at ? at + used : nullptr;
        used += (bytes + 255) & ~(size_t)255;
        return p;
    }
};

unsigned grid_of(int64_t threads) { return (unsigned)std::min<int64_t>((threads + 255) / 256, 1 << 16); }

template <int DT>
hipError_t join_as(const LinearOut& e, const float* partial, int64_t rows, int N, int splits, hipStream_t s)
{
    hipLaunchKernelGGL((linear_join<DT>), dim3((unsigned)((rows * N + 255) / 256)), dim3(256), 0, s, e, partial, rows, N, splits);
    return hipGetLastError();
}
hipError_t join(int dtype, const LinearOut& e, const float* partial, int64_t rows, int N, int splits, hipStream_t s)
{
    return dtype == CONV_F32 ? join_as<CONV_F32>(e, partial, rows, N, splits, s)
                             : dtype == CONV_F16 ? join_as<CONV_F16>(e, partial, rows, N, splits, s) : join_as<CONV_BF16>(e, partial, rows, N, splits, s);
}

// C = A B, in one launch or two, and the join where a reduction is shared.  plane: where A's low part is, 0 if it has one part.
struct Factor {
    const void* p;
    int64_t ld, plane = 0;
};
hipError_t multiply(int dtype, ProductLayout layout, const Factor& a, const Factor& b, int64_t M, int64_t N, int64_t K, const LinearOut& e,
                    const ProductPlan& plan, float* partial, hipStream_t s)
{
    ProductArgs g = {};
    g.a = (const uint16_t*)a.p, g.b = (const uint16_t*)b.p, g.lda = a.ld, g.ldb = b.ld, g.M = M, g.N = N, g.K = K, g.partial = partial;
    g.ksteps = (int)((K + 63) / 64), g.plane_a = a.plane;
    const auto launch = dtype == CONV_F32   ? launch_product_f32
                        : dtype == CONV_F16 ? (a.plane ? launch_product_parts_f16 : launch_product_f16)
                                            : (a.plane ? launch_product_parts_bf16 : launch_product_bf16);
    g.M = plan.rows;
    hipError_t err = launch(g, e, layout, plan.form, plan.splits, s);
    if (err == hipSuccess && plan.splits > 1) err = join(dtype, e, partial, g.M, (int)N, plan.splits, s);
    if (err != hipSuccess || plan.rows == M) return err;
    const int es = dtype_size(dtype);
    LinearOut rest = e;
    rest.out = (char*)e.out + plan.rows * e.ldo * es;
    if (e.pre) rest.pre = (char*)e.pre + plan.rows * e.ldo * es;
    if (e.residual) rest.residual = (const char*)e.residual + plan.rows * e.ldr * es;
    g.a = (const uint16_t*)((const char*)a.p + plan.rows * (layout == LAYOUT_TN ? 1 : a.ld) * es), g.M = M - plan.rows;
    err = launch(g, rest, layout, plan.rest, plan.rest_splits, s);
    return err != hipSuccess || plan.rest_splits == 1 ? err : join(dtype, rest, partial, g.M, (int)N, plan.rest_splits, s);
}
size_t partial_bytes(const ProductPlan& p, int64_t M, int64_t N)
{
    const size_t first = p.splits > 1 ? (size_t)p.splits * p.rows * N * 4 : 0, rest = p.rest_splits > 1 ? (size_t)p.rest_splits * (M - p.rows) * N * 4 : 0;
    return std::max(first, rest);
}

template <int DT, int NB, int RB, int W, int U, bool DIRECT>
hipError_t launch_rows(const LinearRows& g, int splits, hipStream_t s)
{
    constexpr size_t LDS = (size_t)W * (NB + RB) * U * 1024 * (DIRECT ? 2 : 1);
    const hipError_t e = ensure_dynamic_lds((const void*)linear_rows<DT, NB, RB, W, U, DIRECT>, LDS);
    if (e != hipSuccess) return e;
    // gridDim.y is at most 65535, and a launch holds less than 2^32 threads: the rows go in portions
    const int64_t across = (g.N + 16 * NB - 1) / (16 * NB), portion = std::min<int64_t>(65535, std::max<int64_t>(1, (1 << 22) / across)) * (16 * RB);
    for (int64_t skip = 0; skip < g.rows; skip += portion) {
        LinearRows p = g;
        constexpr int ES = sizeof(typename Prec<DT>::elem_t);
        p.rows = std::min(portion, g.rows - skip);
        p.x = (const char*)g.x + skip * g.ldx * ES, p.out.out = (char*)g.out.out + skip * g.out.ldo * ES;
        if (g.out.pre) p.out.pre = (char*)g.out.pre + skip * g.out.ldo * ES;
        if (g.out.residual) p.out.residual = (const char*)g.out.residual + skip * g.out.ldr * ES;
        hipLaunchKernelGGL((linear_rows<DT, NB, RB, W, U, DIRECT>), dim3((unsigned)across, (unsigned)((p.rows + 16 * RB - 1) / (16 * RB)), (unsigned)splits),
                           dim3(64 * W), LDS, s, p);
        if (splits > 1) {
            const hipError_t j = join_as<DT>(p.out, g.partial, p.rows, g.N, splits, s);
            if (j != hipSuccess) return j;
        }
    }
    return hipGetLastError();
}
// Waves a workgroup, and 64-byte pieces of a row in a run: what is on its way to a CU is what counts, and LDS holds it.  Long rows: 8 waves, with runs of 256
// bytes where there is about a workgroup a CU (1 x 4096 x 4096 fp16, weights from memory 8.7 -> 8.2 us), else of 128 in two workgroups.  12 waves for 32
// rows were no better (24 x 6752 x 46704 fp32 329 us with 8, 337).
template <int DT, bool DIRECT>
hipError_t launch_rows(const LinearRows& g, const RowsPlan& p, hipStream_t s)
{
    const int64_t bytes = (int64_t)g.K * (int)sizeof(typename Prec<DT>::elem_t);
    const bool narrow = bytes <= 1024, alone = (int64_t)(g.N + 15) / 16 * p.splits <= 384 && bytes >= 4096;
    if constexpr (DT == CONV_F32) {
        if (p.nb > 1) {
            if constexpr (DIRECT) return p.rb == 2 ? launch_rows<DT, 4, 2, 4, 2, DIRECT>(g, p.splits, s) : launch_rows<DT, 4, 4, 4, 2, DIRECT>(g, p.splits, s);
            else return p.rb == 1 ? launch_rows<DT, 2, 1, 4, 4, DIRECT>(g, p.splits, s) : launch_rows<DT, 2, 2, 4, 4, DIRECT>(g, p.splits, s);
        }
    }
    switch (p.rb) {
        case 1:
            if constexpr (DIRECT) {
                if (alone) return launch_rows<DT, 1, 1, 8, 4, DIRECT>(g, p.splits, s);
            }
            return narrow ? launch_rows<DT, 1, 1, 4, 2, DIRECT>(g, p.splits, s) : launch_rows<DT, 1, 1, 8, 2, DIRECT>(g, p.splits, s);
        case 2:
            return narrow ? launch_rows<DT, 1, 2, 4, 2, DIRECT>(g, p.splits, s) : launch_rows<DT, 1, 2, 8, 2, DIRECT>(g, p.splits, s);
        default: return narrow || DIRECT ? launch_rows<DT, 1, 4, 4, 2, DIRECT>(g, p.splits, s) : launch_rows<DT, 1, 4, 8, 2, DIRECT>(g, p.splits, s);
    }
}
template <int DT>
hipError_t launch_rows(const LinearRows& g, const LinearForm& f, hipStream_t s)
{
    return f.direct ? launch_rows<DT, true>(g, f.few, s) : launch_rows<DT, false>(g, f.few, s);
}

// ---- the backward pass ----------------------------------------------------------------------------------------------------

// Rows a workgroup of linear_dz takes: as many as give some 1024 workgroups, 64 at least.
int64_t dz_rows(int64_t rows, int N)
{
    const int64_t across = (N + 255) / 256, parts = std::max<int64_t>(1, std::min<int64_t>((1024 + across - 1) / across, rows / 64));
    return std::max<int64_t>(round_up((rows + parts - 1) / parts, 8), 8);
}
int dz_parts(int64_t rows, int N) { return rows == 0 ? 0 : (int)((rows + dz_rows(rows, N) - 1) / dz_rows(rows, N)); }

// Rows of dz start on lines of 128 bytes in 16-bit types: a step's 128 bytes of a row would lie in two.
int64_t dz_stride(int N, int dtype) { return dtype == CONV_F32 ? N : round_up(N, 64); }

// Parts of dz: two where the activation's slope is none of 0 and 1.
int dz_parts_of(int act, int dtype) { return dtype != CONV_F32 && act >= ACT_GELU ? 2 : 1; }

struct BwdSpace {
    void* dz;
    int64_t plane;  // elements of a part
    float *sums, *partial;
    size_t bytes;
};
// dz has a place of its own whatever the call needs: the sizes alone say how much a caller keeps.
BwdSpace bwd_space(const LinearArgs& a, int dtype, void* ws)
{
    BwdSpace s = {};
    Carve c(ws);
    const int parts = dz_parts_of(a.act, dtype);
    s.plane = a.rows * dz_stride(a.N, dtype);
    s.dz = c.take((size_t)parts * s.plane * dtype_size(dtype));
    s.sums = (float*)c.take((size_t)dz_parts(a.rows, a.N) * a.N * 4);
    size_t most = 0;
    for (const bool direct : {true, false}) {
        most = std::max(most, partial_bytes(plan_product(a.rows, a.K, a.N, dtype, direct, true, parts), a.rows, a.K));
        most = std::max(most, partial_bytes(plan_product(a.N, a.K, a.rows, dtype, direct, true, parts), a.N, a.K));
    }
    s.partial = (float*)c.take(most);
    s.bytes = c.used;
    return s;
}

template <int DT>
hipError_t launch_dz(const LinearArgs& a, void* dz, int64_t ldz, int64_t plane, float* sums, hipStream_t s)
{
    const int64_t each = dz_rows(a.rows, a.N);
    const int parts = dz_parts(a.rows, a.N);
    const dim3 grid((unsigned)(((dz ? ldz : a.N) + 255) / 256), (unsigned)parts);
    float* const at = !a.dbias ? nullptr : parts == 1 ? a.dbias : sums;
    const auto kernel = !dz ? linear_dz<DT, 0> : plane && DT != CONV_F32 ? linear_dz<DT, DT == CONV_F32 ? 1 : 2> : linear_dz<DT, 1>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a.dout, a.pre_in, a.ldo, a.rows, a.N, a.act, dz, ldz, plane, at, each);
    if (a.dbias && parts > 1) hipLaunchKernelGGL(linear_sums, dim3((unsigned)((a.N + 31) / 32)), dim3(1024), 0, s, sums, parts, a.N, a.dbias);
    return hipGetLastError();
}

}  // namespace

// (the larger of what operands on 16 bytes and others need: what a caller keeps depends on the sizes alone)
size_t linear_fwd_workspace(int64_t rows, int N, int K, int dtype)
{
    if (rows == 0) return 0;
    size_t most = 0;
    for (const bool direct : {true, false}) {
        const LinearForm f = form_of(rows, N, K, dtype, direct);
        size_t n = 0;
        if (f.rows) n = f.few.splits > 1 ? (size_t)f.few.splits * rows * N * 4 : 0;
        else n = partial_bytes(f.tiles, rows, N);
        most = std::max(most, n);
    }
    return most;
}
size_t linear_bwd_workspace(int64_t rows, int N, int K, int act, int dtype)
{
    if (rows == 0) return 0;
    LinearArgs a = {};
    a.rows = rows, a.N = N, a.K = K, a.act = act;
    return bwd_space(a, dtype, nullptr).bytes;
}

hipError_t launch_linear_fwd(const LinearArgs& a, int dtype, hipStream_t s)
{
    const int es = dtype_size(dtype);
    const LinearForm f = form_of(a.rows, a.N, a.K, dtype, on_16(a.x, a.ldx, es) && on_16(a.w, a.ldw, es));
    const LinearOut out = {a.bias, a.residual, a.pre, a.out, a.ldr, a.ldo, a.act};
    if (f.rows) {
        const LinearRows g = {a.x, a.w, a.ldx, a.ldw, a.rows, a.N, a.K, out, (float*)a.ws};
        return dtype == CONV_F32 ? launch_rows<CONV_F32>(g, f, s) : dtype == CONV_F16 ? launch_rows<CONV_F16>(g, f, s) : launch_rows<CONV_BF16>(g, f, s);
    }
    return multiply(dtype, LAYOUT_NT, {a.x, a.ldx}, {a.w, a.ldw}, a.rows, a.N, a.K, out, f.tiles, (float*)a.ws, s);
}

hipError_t launch_linear_bwd(const LinearArgs& a, int dtype, hipStream_t s)
{
    const int es = dtype_size(dtype);
    if (a.rows == 0) {
        if (a.dw) hipLaunchKernelGGL(linear_zero, dim3(grid_of((int64_t)a.N * a.K)), dim3(256), 0, s, (char*)a.dw, a.ldw * es, (int64_t)a.N, (int64_t)a.K * es);
        if (a.dbias) hipLaunchKernelGGL(linear_zero, dim3(grid_of(a.N)), dim3(256), 0, s, (char*)a.dbias, (int64_t)a.N * 4, (int64_t)1, (int64_t)a.N * 4);
        return hipGetLastError();
    }
    const BwdSpace space = bwd_space(a, dtype, a.ws);
    const Factor x = {a.x, a.ldx}, w = {a.w, a.ldw};
    Factor dz = {a.dout, a.ldo};
    // dout is dz where there is no activation and its rows start on 16 bytes (in fp32 anywhere)
    const bool make = (a.dx || a.dw) && (a.act || (dtype != CONV_F32 && !on_16(a.dout, a.ldo, es)));
    const int parts = dz_parts_of(a.act, dtype);
    if (make) dz = {space.dz, dz_stride(a.N, dtype), parts == 2 ? space.plane : 0};
    if (make || a.dbias) {
        void* const to = make ? space.dz : nullptr;
        const hipError_t e = dtype == CONV_F32 ? launch_dz<CONV_F32>(a, to, dz.ld, dz.plane, space.sums, s)
                                               : dtype == CONV_F16 ? launch_dz<CONV_F16>(a, to, dz.ld, dz.plane, space.sums, s) : launch_dz<CONV_BF16>(a, to, dz.ld, dz.plane, space.sums, s);
        if (e != hipSuccess) return e;
    }
    if (a.dx) {
        const ProductPlan p = plan_product(a.rows, a.K, a.N, dtype, on_16(w.p, w.ld, es) && on_16(dz.p, dz.ld, es), true, parts);
        const hipError_t e = multiply(dtype, LAYOUT_NN, dz, w, a.rows, a.K, a.N, {nullptr, nullptr, nullptr, a.dx, 0, a.ldx, ACT_NONE}, p, space.partial, s);
        if (e != hipSuccess) return e;
    }
    if (a.dw) {
        const ProductPlan p = plan_product(a.N, a.K, a.rows, dtype, on_16(x.p, x.ld, es) && on_16(dz.p, dz.ld, es), true, parts);
        const hipError_t e = multiply(dtype, LAYOUT_TN, dz, x, a.N, a.K, a.rows, {nullptr, nullptr, nullptr, a.dw, 0, a.ldw, ACT_NONE}, p, space.partial, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int linear_form_name(const LinearArgs& a, int dtype, int which, char* buf, size_t n)
{
    static const char* const tiles[] = {"tile64x64", "tile128x128", "tile256x256", "tile192x192", "tile64x64_any", "tile128x128_any"};
    const int es = dtype_size(dtype);
    const bool x16 = on_16(a.x, a.ldx, es), w16 = on_16(a.w, a.ldw, es);
    const int parts = which ? dz_parts_of(a.act, dtype) : 1;
    ProductPlan p;
    if (which == 0) {
        const LinearForm f = form_of(a.rows, a.N, a.K, dtype, x16 && w16);
        if (f.rows) {
            char outputs[8] = "";
            if (f.few.nb > 1) std::snprintf(outputs, sizeof(outputs), "x%d", 16 * f.few.nb);
            const int len = std::snprintf(buf, n, "rows%d%s%s", 16 * f.few.rb, outputs, f.direct ? "" : "_any");
            return f.few.splits > 1 && len > 0 && (size_t)len < n ? std::snprintf(buf + len, n - len, "_split%d", f.few.splits) : len;
        }
        p = f.tiles;
    } else if (which == 1) {
        p = plan_product(a.rows, a.K, a.N, dtype, w16, true, parts);
    } else {
        p = plan_product(a.N, a.K, a.rows, dtype, x16, true, parts);
    }
    auto one = [&](char* to, size_t room, ProductForm form, int splits) {
        const char* const name = dtype == CONV_F32 && form == P256 ? "tile256x128" : tiles[form];
        const char* const kind = dtype == CONV_F32 ? "split_" : parts == 2 ? "parts_" : "";
        return splits > 1 ? std::snprintf(to, room, "%s%s_split%d", kind, name, splits) : std::snprintf(to, room, "%s%s", kind, name);
    };
    const int len = one(buf, n, p.form, p.splits);
    if (p.rows == (which == 2 ? a.N : a.rows) || len < 0 || (size_t)len + 1 >= n) return len;
    buf[len] = '+';
    return len + 1 + one(buf + len + 1, n - len - 1, p.rest, p.rest_splits);
}

}  // namespace convfwd
