// Log probabilities of given tokens with entropy and the likeliest alternatives, and their gradient.
//
// Forward, one pass over the logits: every thread keeps the running maximum m of what it has read, s = sum e^(x-m) and
// sd = sum e^(x-m) (x-m); when m grows to m', s' = c s and sd' = c (sd + s (m-m')) with c = e^(m-m').  Threads, and the
// workgroups that share a row, are joined by the same rule; lse = m + log s, entropy = log s - sd / s.
//
// Alternatives are found without sorting: a thread also keeps its largest 16-byte piece (value, and the lower piece where values
// are equal).  The `top`-th largest of 64 such maxima is a bound below which no alternative lies, and only about `top` threads
// hold anything above it; their pieces are read once more (from cache), what reaches the bound goes to a list in LDS, and its
// elements are ranked by counting.  For logits in no particular order the list has little more than `top` entries.  Rows where it
// would overflow, and rows with a NaN or +inf, take the alternatives one by one instead, a pass over the row for each.
#include <algorithm>

#include "rows_common.h"

namespace convfwd {

namespace {

constexpr float kInf = __builtin_inff();
constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504f;
constexpr int kMostTop = 64;

// Whole numbers in the order of the floats: -0 equals +0, a NaN is above everything.
__device__ __forceinline__ uint32_t order_of(float x)
{
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o)
{
    return __builtin_bit_cast(float, (o & 0x80000000u) ? (o == 0xFFFFFFFFu ? 0x7FC00000u : o & 0x7FFFFFFFu) : ~o);
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

// e^d; d * log2 e is rounded once, so the result is off by |d| units of 2^-24 at most, and 0 below 2^-126
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// Sums over part of a row, relative to e^m.  m starts at the lowest number, not at -inf, so that m - m is a number.
struct Part {
    float m, s, sd;
};
__device__ __forceinline__ void rebase(Part& p, float m)
{
    const float d = fmaxf(p.m - m, -1e20f), c = exp_of(d);
    p.sd = c * __builtin_fmaf(p.s, d, p.sd);
    p.s *= c;
    p.m = m;
}
template <int VEC>
__device__ __forceinline__ void add_piece(Part& p, const float (&x)[VEC])
{
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float d = x[i] - p.m, e = exp_of(d);
        p.s += e;
        p.sd = __builtin_fmaf(e, fmaxf(d, -1e20f), p.sd);  // -inf adds 0 * -1e20
    }
}
template <int VEC>
__device__ __forceinline__ float piece_max(const float (&x)[VEC])
{
    float m = fmaxf(x[0], x[1]);
#pragma unroll
    for (int i = 2; i < VEC; ++i) m = fmaxf(m, x[i]);
    return m;
}

template <int W>
__device__ __forceinline__ Part block_join(Part p, float* lds)  // lds: 2 * W floats
{
    const float m = block_reduce<W, OpMax>(p.m, lds);
    rebase(p, m);
    p.s = lanes_reduce<64, OpSum>(p.s);
    p.sd = lanes_reduce<64, OpSum>(p.sd);
    if constexpr (W > 1) {
        __syncthreads();
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) lds[wave] = p.s, lds[W + wave] = p.sd;
        __syncthreads();
        p.s = lds[0], p.sd = lds[W];
#pragma unroll
        for (int i = 1; i < W; ++i) p.s += lds[i], p.sd += lds[W + i];
    }
    return p;
}

// The rank-th largest (from 0) of 64 keys, one a lane; keys that are not 0 are distinct.  0 if there are not as many.
__device__ __forceinline__ uint64_t nth_of_wave(uint64_t key, int rank)
{
    int before = 0;
    const uint32_t lo = (uint32_t)key, hi = (uint32_t)(key >> 32);
#pragma unroll 8
    for (int l = 0; l < 64; ++l) {
        const uint64_t o = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)lo, l);
        before += o > key;
    }
    const uint64_t hit = __ballot(before == rank && key != 0);
    if (!hit) return 0;
    const int l = __builtin_ctzll(hit);
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)lo, l);
}

// The first `top` of n keys in LDS, in order, to best[0..top) (0 where there are fewer): an element's place is the number of greater ones.
template <int NT>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, uint64_t* best, int top)
{
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t k = keys[i];
        int r = 0;
        for (int j = 0; j < n; ++j) r += keys[j] > k;
        if (r < top) best[r] = k;
    }
}

struct RowResult {
    float lse, h;
    bool empty;
};
__device__ __forceinline__ RowResult result_of(const Part& p)
{
    RowResult r;
    r.empty = p.s == 0.0f;
    const float l = logf(p.s);
    r.lse = p.m + l, r.h = l - p.sd / p.s;
    if (r.empty) r.lse = -kInf, r.h = 0.0f;
    return r;
}

// What a row's results are written from, by the workgroup that has them.
template <int DT, int NT>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t row, const Part& p, const uint64_t* best)
{
    typedef typename Prec<DT>::elem_t elem_t;
    const RowResult r = result_of(p);
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = r.lse;
        if (a.entropy) a.entropy[row] = r.h;
        if (a.logp) {
            const int64_t t = a.target[row];
            float v = 0.0f;
            if (t >= a.cols) v = __builtin_nanf("");
            else if (t >= 0) v = r.empty ? -kInf : Prec<DT>::to_f32(((const elem_t*)a.x)[row * a.ldx + t]) - r.lse;
            a.logp[row] = v;
        }
    }
    for (int i = threadIdx.x; i < a.top; i += NT) {
        const uint64_t k = best[i];
        a.top_id[row * a.top + i] = (int64_t)index_of(k);
        a.top_logp[row * a.top + i] = r.empty ? -kInf : value_of((uint32_t)(k >> 32)) - r.lse;
    }
}

// Partial results of a row that several workgroups share: `splits` parts, then `splits` lists of `top` keys (16 bytes each row's start).
__host__ __device__ __forceinline__ size_t part_bytes(int top) { return 16 + 8 * (size_t)((top + 1) & ~1); }

// One row, or one of `splits` shares of `share` pieces of it, a workgroup of W waves.  TOP: alternatives are asked for.
template <int DT, int W, bool TOP>
__global__ __launch_bounds__(64 * W) void logprob_rows(LogprobArgs a, int splits, int share)
{
    typedef typename Prec<DT>::elem_t elem_t;
    typedef Piece<DT> P;
    constexpr int VEC = P::VEC, NT = 64 * W, U = 4;
    constexpr int LIST = W == 1 ? 640 : 1024;  // at least 64 pieces of 8: rows of so few pieces go there whole
    __shared__ float red[2 * W];
    __shared__ uint64_t maxima[TOP ? NT : 1], list[TOP ? LIST : 1], best[TOP ? kMostTop : 1], bound;
    __shared__ uint16_t winner[TOP ? NT : 1];
    __shared__ int listed, winners;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int full = a.cols / VEC, rest = a.cols % VEC;  // whole pieces, and elements behind the last
    const int v0 = blockIdx.y * share, v1 = min(full, v0 + share);
    const bool has_rest = rest && blockIdx.y == splits - 1;

    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const elem_t* x = (const elem_t*)a.x + row * a.ldx;
        Part p = {kLowest, 0.0f, 0.0f};
        float most = -kInf;
        int at = -1;  // the piece with `most`
        auto rest_piece = [&](float (&f)[VEC]) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = i < rest ? Prec<DT>::to_f32(x[(int64_t)full * VEC + (i < rest ? i : 0)]) : -kInf;
        };
        auto note = [&](float m, int v) {
            if (TOP && m > most) most = m, at = v;
        };
        int v = v0 + tid;
        for (; v + (U - 1) * NT < v1; v += U * NT) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = P::raw(x + (int64_t)(v + u * NT) * VEC);
            float f[U][VEC], m[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                P::widen(raw[u], f[u]);
                m[u] = piece_max(f[u]);
                note(m[u], v + u * NT);
            }
            const float mm = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
            if (mm > p.m) rebase(p, mm);
#pragma unroll
            for (int u = 0; u < U; ++u) add_piece(p, f[u]);
        }
        for (; v < v1 || (has_rest && v == full); v += NT) {
            float f[VEC];
            if (v < v1) P::widen(P::raw(x + (int64_t)v * VEC), f);
            else rest_piece(f);
            const float m = piece_max(f);
            note(m, v);
            if (m > p.m) rebase(p, m);
            add_piece(p, f);
        }
        __syncthreads();  // the previous row's LDS is free
        p = block_join<W>(p, red);
        if constexpr (TOP) {
            const int end = v1 + (has_rest ? 1 : 0);  // pieces of this workgroup, the last one short
            if (at < 0 && v0 + tid < end) at = v0 + tid;  // nothing but -inf
            const uint64_t mine = at < 0 ? 0 : key_of(most, (uint32_t)at);
            maxima[tid] = mine;
            for (int i = tid; i < kMostTop; i += NT) best[i] = 0;
            if (tid == 0) listed = 0, winners = 0;
            __syncthreads();
            if (wave == 0) {
                uint64_t k = maxima[lane];
#pragma unroll
                for (int w = 1; w < W; ++w) k = maxima[w * 64 + lane] > k ? maxima[w * 64 + lane] : k;
                const uint64_t b = nth_of_wave(k, a.top - 1);
                if (lane == 0) bound = b;
            }
            __syncthreads();
            const uint64_t b = bound;
            const uint32_t b_order = (uint32_t)(b >> 32), b_piece = b ? index_of(b) : 0xFFFFFFFFu;
            const bool odd = !(p.s >= 0.0f);  // a NaN or an infinity
            if (!odd) {
                if (mine && mine >= b) winner[atomicAdd(&winners, 1)] = (uint16_t)tid;
                __syncthreads();
                const int n = winners;
                for (int i = wave; i < n; i += W) {
                    for (int q = v0 + winner[i] + lane * NT; q < end; q += 64 * NT) {
                        float f[VEC];
                        if (q < v1) P::widen(P::raw(x + (int64_t)q * VEC), f);
                        else rest_piece(f);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            const uint32_t o = order_of(f[e]);
                            if ((o > b_order || (o == b_order && (uint32_t)q <= b_piece)) && q * VEC + e < a.cols) {
                                const int to = atomicAdd(&listed, 1);
                                if (to < LIST) list[to] = key_of(f[e], (uint32_t)(q * VEC + e));
                            }
                        }
                    }
                }
                __syncthreads();
            }
            if (!odd && listed <= LIST) {
                rank_keys<NT>(list, listed, best, a.top);
            } else {
                const int j0 = v0 * VEC, j1 = has_rest ? a.cols : v1 * VEC;
                uint64_t last = ~0ull;
                for (int i = 0; i < a.top; ++i) {
                    uint64_t k = 0;
                    for (int j = j0 + tid; j < j1; j += NT) {
                        const uint64_t c = key_of(Prec<DT>::to_f32(x[j]), (uint32_t)j);
                        if (c < last && c > k) k = c;
                    }
                    k = wave_max(k);
                    __syncthreads();
                    if (lane == 0) list[wave] = k;
                    __syncthreads();
                    k = list[0];
#pragma unroll
                    for (int w = 1; w < W; ++w) k = list[w] > k ? list[w] : k;
                    if (tid == 0) best[i] = k;
                    last = k;
                }
            }
            __syncthreads();
        }
        if (splits == 1) {
            write_row<DT, NT>(a, row, p, best);
        } else {
            char* ws = (char*)a.ws + (size_t)row * splits * part_bytes(a.top);
            if (tid == 0) ((float4*)ws)[blockIdx.y] = make_float4(p.m, p.s, p.sd, 0.0f);
            uint64_t* keys = (uint64_t*)(ws + 16 * (size_t)splits) + (size_t)blockIdx.y * a.top;
            for (int i = tid; i < a.top; i += NT) keys[i] = best[i];
        }
    }
}

constexpr int kMostSplits = 64;

// Joins the `splits` parts of a row: a workgroup of four waves a row.
template <int DT>
__global__ __launch_bounds__(256) void logprob_join(LogprobArgs a, int splits)
{
    constexpr int NT = 256;
    __shared__ float red[8];
    __shared__ uint64_t maxima[NT], list[kMostSplits * kMostTop], best[kMostTop], bound;
    __shared__ int listed;
    const int tid = threadIdx.x, lane = tid & 63;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const char* ws = (const char*)a.ws + (size_t)row * splits * part_bytes(a.top);
        Part p = {kLowest, 0.0f, 0.0f};
        if (tid < splits) {
            const float4 f = ((const float4*)ws)[tid];
            p.m = f.x, p.s = f.y, p.sd = f.z;
        }
        __syncthreads();
        p = block_join<4>(p, red);
        if (a.top) {
            const uint64_t* keys = (const uint64_t*)(ws + 16 * (size_t)splits);
            const int n = splits * a.top;
            uint64_t most = 0;
            for (int i = tid; i < n; i += NT) most = keys[i] > most ? keys[i] : most;
            maxima[tid] = most;
            for (int i = tid; i < kMostTop; i += NT) best[i] = 0;
            if (tid == 0) listed = 0;
            __syncthreads();
            if (tid < 64) {
                uint64_t k = maxima[lane];
#pragma unroll
                for (int w = 1; w < 4; ++w) k = maxima[w * 64 + lane] > k ? maxima[w * 64 + lane] : k;
                const uint64_t b = nth_of_wave(k, a.top - 1);
                if (lane == 0) bound = b;
            }
            __syncthreads();
            const uint64_t b = bound ? bound : 1;  // 0 stands for no element
            for (int i = tid; i < n; i += NT)
                if (keys[i] >= b) list[atomicAdd(&listed, 1)] = keys[i];
            __syncthreads();
            rank_keys<NT>(list, listed, best, a.top);
            __syncthreads();
        }
        write_row<DT, NT>(a, row, p, best);
    }
}

// The gradient: a piece of 16 bytes is read, and written, by one thread.  `per_row` threads (a power of two up to 256) share a row,
// or, for longer rows, a workgroup has 1024 pieces of one.  x - lse = log p, so with c = g_logp + g_entropy (log p + entropy) every
// element is -p c, and the target's g_logp more.
template <int DT>
__global__ __launch_bounds__(256) void logprob_bwd_rows(LogprobArgs a, int per_row)
{
    typedef typename Prec<DT>::elem_t elem_t;
    typedef Piece<DT> P;
    constexpr int VEC = P::VEC, U = 4;
    const int rows_here = 256 / per_row, l = threadIdx.x & (per_row - 1);
    const int pieces = (a.cols + VEC - 1) / VEC, first = blockIdx.y * (per_row * U);
    for (int64_t row = (int64_t)blockIdx.x * rows_here + threadIdx.x / per_row; row < a.rows; row += (int64_t)gridDim.x * rows_here) {
        const elem_t* x = (const elem_t*)a.x + row * a.ldx;
        elem_t* dx = (elem_t*)a.dx + row * a.ldg;
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t j = (int64_t)(first + u * per_row + l) * VEC;
            if (j + VEC <= a.cols) {
                raw[u] = P::raw(x + j);
            } else {
                elem_t e[VEC];
#pragma unroll
                for (int k = 0; k < VEC; ++k) e[k] = j + k < a.cols ? x[j + k] : (elem_t)0;
                __builtin_memcpy(&raw[u], e, 16);
            }
        }
        const float lse = a.lse[row];
        const bool empty = lse == -kInf;
        const int64_t t = a.g_logp ? a.target[row] : -1;
        float g = t >= 0 ? a.g_logp[row] : 0.0f;
        if (t >= a.cols) g = __builtin_nanf("");
        const float gh = a.g_entropy ? a.g_entropy[row] : 0.0f, h = a.g_entropy ? a.entropy[row] : 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = first + u * per_row + l;
            if (q >= pieces) break;
            const int64_t j = (int64_t)q * VEC;
            float f[VEC];
            P::widen(raw[u], f);
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const float lp = f[k] - lse, p = exp_of(lp);
                f[k] = -p * __builtin_fmaf(gh, fmaxf(lp, -1e20f) + h, g);  // -inf: p is 0
            }
            if (t >= j && t < j + VEC) {
#pragma unroll
                for (int k = 0; k < VEC; ++k) f[k] += t == j + k ? g : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < VEC; ++k) f[k] = empty ? 0.0f : f[k];
            const uint4 out = P::narrow(f);
            if (j + VEC <= a.cols) {
                P::put(dx + j, out);
            } else {
                elem_t e[VEC];
                __builtin_memcpy(e, &out, 16);
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    if (j + k < a.cols) dx[j + k] = e[k];
            }
        }
    }
}

// How a row is shared: one workgroup where the rows alone fill the GPU (two workgroups a CU), else as many as leave each of them
// two pieces a thread, up to 64.
struct Shares {
    int waves, splits, share;
};
Shares shares_of(int64_t rows, int cols, int dtype)
{
    const int vec = dtype == CONV_F32 ? 4 : 8, full = cols / vec;
    Shares s;
    s.waves = full <= 256 ? 1 : full <= 1024 ? 4 : 8;
    int64_t want = (512 + rows - 1) / std::max<int64_t>(rows, 1);
    want = std::min<int64_t>(want, kMostSplits);
    if (want > 1 && full > 1024) {
        s.waves = 4;
        want = std::min<int64_t>(want, full / 512);
    } else {
        want = 1;
    }
    s.share = (int)((full + want - 1) / want);
    s.splits = s.share ? (full + s.share - 1) / s.share : 1;
    if (s.splits < 1) s.splits = 1;
    return s;
}

template <int DT, int W>
void launch_w(LogprobArgs& a, const Shares& sh, hipStream_t s)
{
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, 1 << 18), (unsigned)sh.splits), block(64 * W);
    if (a.top) hipLaunchKernelGGL((logprob_rows<DT, W, true>), grid, block, 0, s, a, sh.splits, sh.share);
    else hipLaunchKernelGGL((logprob_rows<DT, W, false>), grid, block, 0, s, a, sh.splits, sh.share);
}

template <int DT>
hipError_t fwd(LogprobArgs& a, hipStream_t s)
{
    const Shares sh = shares_of(a.rows, a.cols, DT);
    if (sh.waves == 1) launch_w<DT, 1>(a, sh, s);
    else if (sh.waves == 4) launch_w<DT, 4>(a, sh, s);
    else launch_w<DT, 8>(a, sh, s);
    if (sh.splits > 1) hipLaunchKernelGGL((logprob_join<DT>), dim3((unsigned)a.rows), dim3(256), 0, s, a, sh.splits);
    return hipGetLastError();
}

}  // namespace

size_t logprob_workspace(int64_t rows, int cols, int top, int dtype)
{
    const Shares sh = shares_of(rows, cols, dtype);
    return sh.splits > 1 ? (size_t)rows * sh.splits * part_bytes(top) : 0;
}

hipError_t launch_logprob_fwd(LogprobArgs& a, int dtype, hipStream_t s)
{
    return dtype == CONV_F32 ? fwd<CONV_F32>(a, s) : dtype == CONV_F16 ? fwd<CONV_F16>(a, s) : fwd<CONV_BF16>(a, s);
}

template <int DT>
static hipError_t bwd(const LogprobArgs& a, hipStream_t s)
{
    constexpr int VEC = Piece<DT>::VEC;
    const int pieces = (a.cols + VEC - 1) / VEC;
    int per_row = 4;  // threads a row: four pieces a thread, up to a workgroup
    while (per_row < 256 && per_row * 4 < pieces) per_row *= 2;
    const int64_t blocks = (a.rows + 256 / per_row - 1) / (256 / per_row);
    const dim3 grid((unsigned)std::min<int64_t>(blocks, 1 << 20), (unsigned)((pieces + per_row * 4 - 1) / (per_row * 4)));
    hipLaunchKernelGGL((logprob_bwd_rows<DT>), grid, dim3(256), 0, s, a, per_row);
    return hipGetLastError();
}

hipError_t launch_logprob_bwd(LogprobArgs& a, int dtype, hipStream_t s)
{
    return dtype == CONV_F32 ? bwd<CONV_F32>(a, s) : dtype == CONV_F16 ? bwd<CONV_F16>(a, s) : bwd<CONV_BF16>(a, s);
}

}  // namespace convfwd
