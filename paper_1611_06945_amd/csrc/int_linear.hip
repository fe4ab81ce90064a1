// Matrix product in 8-bit integers with scales for each row and output channel.
#include <algorithm>

#include "rows_common.h"

namespace convfwd {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;

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

// A wave 16 channels x 16 rows, operands from memory straight into registers: any strides.
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

// Tiles of BT rows x BN channels, both operands staged through LDS by loads that write it directly, two stages.
//   * A stage holds 128 bytes of each row; a row's eight 16-byte pieces are stored at piece ^ (row / 2 % 8), by choosing which piece
//     a lane loads: the 16 lanes that LDS serves together then read 16 different groups of four banks.
//   * Rows past the last one, and pieces past the end of the tensor, are read as zeros by the bounds check of the buffer
//     descriptor; the bytes of a row past K belong to what follows and are cleared in one operand on the last step.
template <int WT_, int WN_, int FT_, int FN_>
struct IntTile {
    static constexpr int WT = WT_, WN = WN_, FT = FT_, FN = FN_;  // waves and 32-wide blocks a wave, along rows and channels
    static constexpr int BT = 32 * WT * FT, BN = 32 * WN * FN, NT = 64 * WT * WN;
    static constexpr int KB = 128;
    static constexpr int STAGE = (BT + BN) * KB;
    static constexpr size_t LDS = 2 * STAGE;
    static constexpr int LA = BT * 8 / NT, LW = BN * 8 / NT;  // 16-byte loads a thread and stage
};

template <int DT, typename T>
__global__ __launch_bounds__(T::NT) void int_linear_tiles(IntLinearArgs g, int tiles_t, int tiles_n)
{
    typedef typename Prec<DT>::elem_t elem_t;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
    const int64_t rows_here = min((int64_t)T::BT, g.rows - t0);
    const int outs_here = min(T::BN, g.N - n0);
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(g.a + t0 * g.lda, (uint32_t)((rows_here - 1) * g.lda + Kr));
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(g.w + (int64_t)n0 * g.ldw, (uint32_t)((outs_here - 1) * g.ldw + Kr));
    uint32_t aoff[T::LA], woff[T::LW];
#pragma unroll
    for (int i = 0; i < T::LA; ++i) {
        const int p = i * T::NT + tid, row = p >> 3;
        aoff[i] = (uint32_t)row * (uint32_t)g.lda + (((p & 7) ^ ((row >> 1) & 7)) << 4);
    }
#pragma unroll
    for (int i = 0; i < T::LW; ++i) {
        const int p = i * T::NT + tid, row = p >> 3;
        woff[i] = (uint32_t)row * (uint32_t)g.ldw + (((p & 7) ^ ((row >> 1) & 7)) << 4);
    }
    auto stage = [&](int buf, int k0) {
        char* base = smem + buf * T::STAGE + wave * 1024;
#pragma unroll
        for (int i = 0; i < T::LA; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(base + i * T::NT * 16), 16, (int)(aoff[i] + k0), 0, 0, 0);
#pragma unroll
        for (int i = 0; i < T::LW; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_void*)(base + T::BT * T::KB + i * T::NT * 16), 16, (int)(woff[i] + k0), 0, 0, 0);
    };
    int frag[4];  // LDS offset of this lane's piece for each step of 32 bytes, without the block
#pragma unroll
    for (int s = 0; s < 4; ++s) frag[s] = (lane & 31) * T::KB + (((s * 2 + (lane >> 5)) ^ ((lane >> 1) & 7)) << 4);

    i32x16 acc[T::FN][T::FT];
#pragma unroll
    for (int i = 0; i < T::FN; ++i)
#pragma unroll
        for (int j = 0; j < T::FT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;

    const int steps = (g.K + T::KB - 1) / T::KB;
    auto multiply = [&](int buf, int left, auto last) {
        const char* pa = smem + buf * T::STAGE + wt * T::FT * 32 * T::KB;
        const char* pw = smem + buf * T::STAGE + (T::BT + wn * T::FN * 32) * T::KB;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            i32x4 av[T::FT], wv[T::FN];
#pragma unroll
            for (int i = 0; i < T::FN; ++i) {
                wv[i] = *(const i32x4*)(pw + frag[s] + i * 32 * T::KB);
                if constexpr (decltype(last)::value) wv[i] = first_bytes(wv[i], left - (s * 2 + (lane >> 5)) * 16);
            }
#pragma unroll
            for (int j = 0; j < T::FT; ++j) av[j] = *(const i32x4*)(pa + frag[s] + j * 32 * T::KB);
#pragma unroll
            for (int i = 0; i < T::FN; ++i)
#pragma unroll
                for (int j = 0; j < T::FT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv[i], av[j], acc[i][j], 0, 0, 0);
        }
    };
    stage(0, 0);
    __syncthreads();
    for (int k = 0; k < steps - 1; ++k) {
        stage((k + 1) & 1, (k + 1) * T::KB);
        multiply(k & 1, 0, std::false_type());
        __syncthreads();  // waits for the loads of this wave as well
    }
    multiply((steps - 1) & 1, g.K - (steps - 1) * T::KB, std::true_type());

    // lane: row (lane & 31) of a block of rows; channels 8 q + 4 (lane / 32) + 0..3 in accumulators 4 q ..  Two q at a time, so that
    // few scales are held; in 16 bits the halves of the wave then trade, and a lane has eight channels in a row: lanes below 32
    // those of q, the others those of q + 1.
    const int half = lane >> 5;
    float sa[T::FT];
    const int64_t t_lane = t0 + wt * T::FT * 32 + (lane & 31);
#pragma unroll
    for (int j = 0; j < T::FT; ++j) sa[j] = g.a_scale[min(t_lane + j * 32, g.rows - 1)];
#pragma unroll
    for (int i = 0; i < T::FN; ++i)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
            const int nb = n0 + (wn * T::FN + i) * 32 + q * 8;
            float sw[8], b[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const int n = min(nb + (r >> 2) * 8 + half * 4 + (r & 3), g.N - 1);
                sw[r] = g.w_scale[n];
                b[r] = g.bias ? g.bias[n] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < T::FT; ++j) {
                const int64_t t = t_lane + j * 32;
                elem_t* out = (elem_t*)g.out + t * g.ldo;
                float v[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = finish(acc[i][j][4 * q + r], sa[j] * sw[r], b[r], g.relu);
                constexpr int LEN = 16 / sizeof(elem_t);
                uint32_t w4[8 / LEN][4];
                int n[8 / LEN];
                if constexpr (DT == CONV_F32) {
                    __builtin_memcpy(w4, v, 32);
                    n[0] = nb + half * 4, n[1] = nb + 8 + half * 4;
                } else {
                    const auto r0 = __builtin_amdgcn_permlane32_swap(Prec<DT>::pack2_from_f32(v[0], v[1]), Prec<DT>::pack2_from_f32(v[4], v[5]), false, false);
                    const auto r1 = __builtin_amdgcn_permlane32_swap(Prec<DT>::pack2_from_f32(v[2], v[3]), Prec<DT>::pack2_from_f32(v[6], v[7]), false, false);
                    w4[0][0] = r0[0], w4[0][1] = r1[0], w4[0][2] = r0[1], w4[0][3] = r1[1];
                    n[0] = nb + half * 8;
                }
#pragma unroll
                for (int c = 0; c < 8 / LEN; ++c) {
                    if (t < g.rows && n[c] + LEN <= g.N) {
                        __builtin_memcpy(out + n[c], w4[c], 16);
                    } else if (t < g.rows) {
                        elem_t e[LEN];
                        __builtin_memcpy(e, w4[c], 16);
#pragma unroll
                        for (int r = 0; r < LEN; ++r)
                            if (n[c] + r < g.N) out[n[c] + r] = e[r];
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
}

typedef IntTile<2, 4, 4, 2> Tile256;  // 256 x 256
typedef IntTile<2, 2, 2, 2> Tile128;  // 128 x 128

template <int DT, typename T>
hipError_t launch_tiles(const IntLinearArgs& g, hipStream_t s)
{
    const void* f = (const void*)int_linear_tiles<DT, T>;
    const hipError_t e = ensure_dynamic_lds(f, T::LDS);
    if (e != hipSuccess) return e;
    const int tt = (int)((g.rows + T::BT - 1) / T::BT), tn = (g.N + T::BN - 1) / T::BN;
    hipLaunchKernelGGL((int_linear_tiles<DT, T>), dim3((unsigned)(tt * tn)), dim3(T::NT), T::LDS, s, g, tt, tn);
    return hipGetLastError();
}

template <int DT>
hipError_t launch(IntLinearArgs& g, hipStream_t s)
{
    // offsets within a tile are 32 bits
    const int64_t most = std::max(g.lda, g.ldw);
    const int64_t tiles = ((g.rows + 255) / 256) * ((g.N + 255) / 256);
    if (most < (1 << 23) && g.rows > 64 && tiles < (1 << 20)) {
        if (tiles >= 192) return launch_tiles<DT, Tile256>(g, s);
        return launch_tiles<DT, Tile128>(g, s);
    }
    const int64_t nt = (g.rows + 15) / 16;
    const dim3 block(256);
    // gridDim.y is at most 65535: the rows go in portions
    for (int64_t t = 0; t < nt; t += 65535) {
        IntLinearArgs p = g;
        const int64_t skip = t * 16, left = g.rows - skip;
        p.rows = left < 65535 * 16 ? left : 65535 * 16;
        p.a += skip * g.lda, p.a_scale += skip, p.out = (char*)g.out + skip * g.ldo * dtype_size(DT);
        const dim3 grid((unsigned)((g.N + 63) / 64), (unsigned)((p.rows + 15) / 16));
        hipLaunchKernelGGL((int_linear_tile16<DT>), grid, block, 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace

size_t int_linear_workspace(int64_t rows, int N, int K) { return 0; }

hipError_t launch_int_linear(IntLinearArgs& g, int dtype, hipStream_t s)
{
    return dtype == CONV_F32 ? launch<CONV_F32>(g, s) : dtype == CONV_F16 ? launch<CONV_F16>(g, s) : launch<CONV_BF16>(g, s);
}

}  // namespace convfwd
