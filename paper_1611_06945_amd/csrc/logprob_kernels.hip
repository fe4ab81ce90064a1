// Log probabilities of given tokens with entropy and the likeliest alternatives, and their gradient.
//
// Forward, one pass over the logits: every thread keeps the running maximum m of what it has read, s = sum e^(x-m) and
// sd = sum e^(x-m) (x-m); when m grows to m', s' = c s and sd' = c (sd + s (m-m')) with c = e^(m-m').  Threads, and the
// workgroups that share a row, are joined by the same rule; lse = m + log s, entropy = log s - sd / s.
//
// Alternatives are found without sorting: a thread also keeps its largest 16-byte piece (value, and the lower piece where values
// are equal).  The `top`-th largest of 16 to 128 such maxima is a bound below which no alternative lies, and only about `top` threads
// hold anything above it; their pieces are read once more (from cache), what reaches the bound goes to a list in LDS, and its
// elements are ranked by counting.  For logits in no particular order the list has little more than `top` entries.  Rows where it
// would overflow, and rows with a NaN or +inf, take the alternatives one by one instead, a pass over the row for each (2048 x 50257 bf16
// whose large logits all lie in the pieces of six threads: 2.7 ms with 20 alternatives, 8.5 with 64, instead of 55 and 74 us).
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

// e^d, off by 1.25 |d| units of 2^-24 at most, for the rounding of the product (1) and of log2 e (0.23), and by the instruction's own
// error; 0 below 2^-126
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

__device__ __forceinline__ uint64_t lane_key(uint64_t key, int l)
{
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)key, l);
}
template <int N>
__device__ __forceinline__ uint64_t nth_of_lanes(uint64_t key, int rank)
{
    int before = 0;
#pragma unroll
    for (int l = 0; l < N; ++l) before += lane_key(key, l) > key;
    const uint64_t hit = __ballot(before == rank && key != 0);
    return hit ? lane_key(key, __builtin_ctzll(hit)) : 0;
}
// ... of 128 keys, two a lane
__device__ __forceinline__ uint64_t nth_of_pairs(uint64_t k0, uint64_t k1, int rank)
{
    int before0 = 0, before1 = 0;
#pragma unroll 4
    for (int l = 0; l < 64; ++l) {
        const uint64_t o0 = lane_key(k0, l), o1 = lane_key(k1, l);
        before0 += (o0 > k0) + (o1 > k0);
        before1 += (o0 > k1) + (o1 > k1);
    }
    const uint64_t hit0 = __ballot(before0 == rank && k0 != 0), hit1 = __ballot(before1 == rank && k1 != 0);
    return hit0 ? lane_key(k0, __builtin_ctzll(hit0)) : hit1 ? lane_key(k1, __builtin_ctzll(hit1)) : 0;
}
// A bound for the `top` largest of 128 sets of keys, given each set's largest, two a lane: the top-th largest of these, or, where `top`
// is small beside 16 or 32, of the largest of four or eight of them (fewer comparisons; for keys in no order 5 of 16 let 6 through, 20 of
// 32 31, 64 of 128 89).  Keys that are not 0 are distinct; 0 if there are not as many.  The steps (us with 8 / 9 and with 20 / 21
// alternatives): 2048 x 50257 bf16 46.0 / 46.0 and 54.9 / 55.6, 20 x 1000 fp32 5.8 / 5.9 and 7.8 / 7.9, 1 x 131072 fp32, which has the chain twice,
// 9.7 / 9.9 and 11.7 / 15.6.
__device__ __forceinline__ uint64_t bound_of_wave(uint64_t k0, uint64_t k1, int top)
{
    if (top > 20) return nth_of_pairs(k0, k1, top - 1);
    uint64_t key = k0 > k1 ? k0 : k1;
    uint64_t o = __shfl_xor(key, 32, 64);
    key = o > key ? o : key;
    if (top > 8) return nth_of_lanes<32>(key, top - 1);
    o = __shfl_xor(key, 16, 64);
    key = o > key ? o : key;
    return nth_of_lanes<16>(key, top - 1);
}

// The first `top` of n keys in LDS, in order, to best[0..top): an element's place is the number of greater ones, counted by eight
// lanes.
template <int NT>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, uint64_t* best, int top)
{
    const int part = threadIdx.x & 7;
    for (int i = threadIdx.x >> 3; i < n; i += NT / 8) {
        const uint64_t k = keys[i];
        int r = 0;
        for (int j = part; j < n; j += 8) r += keys[j] > k;
        r += __builtin_amdgcn_mov_dpp(r, 0xB1, 0xF, 0xF, false);   // the eight lanes' counts: quad_perm [1,0,3,2], [2,3,0,1],
        r += __builtin_amdgcn_mov_dpp(r, 0x4E, 0xF, 0xF, false);
        r += __builtin_amdgcn_mov_dpp(r, 0x141, 0xF, 0xF, false);  // row_half_mirror
        if (part == 0 && r < top) best[r] = k;
    }
}

// The sum of `n` over the lanes up to and with this one.
__device__ __forceinline__ int wave_scan(int n)
{
    n += __builtin_amdgcn_update_dpp(0, n, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8: within 16 lanes
    n += __builtin_amdgcn_update_dpp(0, n, 0x112, 0xF, 0xF, false);
    n += __builtin_amdgcn_update_dpp(0, n, 0x114, 0xF, 0xF, false);
    n += __builtin_amdgcn_update_dpp(0, n, 0x118, 0xF, 0xF, false);
    n += __builtin_amdgcn_update_dpp(0, n, 0x142, 0xA, 0xF, false);  // lane 15 to row 1, lane 47 to row 3
    n += __builtin_amdgcn_update_dpp(0, n, 0x143, 0xC, 0xF, false);  // lane 31 to rows 2 and 3
    return n;
}
// Room in a list for `n` entries of each lane, by one addition a wave (left to the compiler, lanes are added one after the other):
// where this lane's begin.  Every lane of the wave calls; `counter` is LDS.
__device__ __forceinline__ int take_room(int n, int* counter)
{
    const int upto = wave_scan(n), total = __builtin_amdgcn_readlane(upto, 63);
    int base = 0;
    if ((threadIdx.x & 63) == 0) base = atomicAdd(counter, total);
    return __builtin_amdgcn_readfirstlane(base) + upto - n;
}

// A log probability is taken as (x - m) - log s, not as x - lse: lse is rounded to units of its own size, and a row of the lowest
// value only would have the log probability 0 throughout.
struct RowResult {
    float m, log_s, lse, h;
    bool empty;
    __device__ __forceinline__ float logp(float x) const { return empty ? -kInf : (x - m) - log_s; }
};
__device__ __forceinline__ RowResult result_of(const Part& p)
{
    RowResult r;
    r.empty = p.s == 0.0f;
    r.m = p.m, r.log_s = logf(p.s);
    r.lse = p.m + r.log_s, r.h = r.log_s - p.sd / p.s;
    if (r.empty) r.lse = -kInf, r.h = 0.0f;
    return r;
}

// The target of a row and its logit (NaN where there is no such column), asked for by one thread ahead of the work on the row.
struct Given {
    bool any;
    float logit;
};
template <int DT>
__device__ __forceinline__ Given given_of(const LogprobArgs& a, int64_t row)
{
    Given g = {false, 0.0f};
    if (a.logp) {
        const int64_t t = a.target[row];
        g.any = t >= 0;
        g.logit = __builtin_nanf("");
        if (t >= 0 && t < a.cols) g.logit = Prec<DT>::to_f32(((const typename Prec<DT>::elem_t*)a.x)[row * a.ldx + t]);
    }
    return g;
}

// Writes a row's results, by the workgroup that has them; `given` counts in thread 0.
template <int NT>
__device__ __forceinline__ void write_row(const LogprobArgs& a, int64_t row, const Given& given, const Part& p, const uint64_t* best)
{
    const RowResult r = result_of(p);
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = r.lse;
        if (a.entropy) a.entropy[row] = r.h;
        // (a logit of NaN without a NaN in the row: no such column)
        if (a.logp) a.logp[row] = !given.any ? 0.0f : given.logit == given.logit ? r.logp(given.logit) : given.logit;
    }
    for (int i = threadIdx.x; i < a.top; i += NT) {
        const uint64_t k = best[i];
        a.top_id[row * a.top + i] = (int64_t)index_of(k);
        a.top_logp[row * a.top + i] = r.logp(value_of((uint32_t)(k >> 32)));
    }
}

// Partial results of a row that several workgroups share: `splits` parts, then `splits` lists of `top` keys (16 bytes each row's start).
__host__ __device__ __forceinline__ size_t part_bytes(int top) { return 16 + 8 * (size_t)((top + 1) & ~1); }

// One row, or one of `splits` shares of `share` pieces of it, a workgroup of W waves.  Pieces begin at multiples of 16 bytes in memory:
// the first and the last of a row can be short (its edges); their elements are a thread's each, stay out of the maxima, and go to
// the list on their own.  HELD: a share is at most U pieces a thread, so that its
// maximum is known before its sums.  TOP: alternatives are asked for.
template <int DT, int W, bool HELD, bool TOP>
__global__ __launch_bounds__(64 * W, TOP ? 1 : 8) void logprob_rows(LogprobArgs a, int splits, int share)
{
    typedef typename Prec<DT>::elem_t elem_t;
    typedef Piece<DT> P;
    constexpr int VEC = P::VEC, NT = 64 * W, U = 4;
    constexpr int LIST = W == 1 ? 640 : 1024;  // at least 64 pieces of 8, and the edges: rows of so few pieces go there whole
    __shared__ float red[2 * W];
    __shared__ uint64_t maxima[TOP ? NT : 1], list[TOP ? LIST : 1], best[TOP ? kMostTop : 1], bound;
    __shared__ uint16_t winner[TOP ? NT : 1];
    __shared__ int listed, winners;
    
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int tid = threadIdx.x;
        const elem_t* const x = (const elem_t*)a.x + row * a.ldx;
        const int shift = (int)(((uintptr_t)x / sizeof(elem_t)) % VEC);  // elements of the row's first 16 bytes that are not its own
        const elem_t* const base = x - shift;                            // element j is base[shift + j]; pieces start at base
        const int whole_end = (int)(((int64_t)a.cols + shift) / VEC);    // whole pieces: shift > 0 .. whole_end
        const int v0 = max((int)blockIdx.y * share, shift > 0 ? 1 : 0), v1 = min(whole_end, ((int)blockIdx.y + 1) * share);
        const int head = shift ? min(VEC - shift, a.cols) : 0, tail = max(whole_end * VEC - shift, head);  // edges: [0, head), [tail, cols)
        // ... an element a thread: the first edge's by the first eight threads of the first share, the last one's by the next eight of the last
        int edge = -1;
        if (tid < 8 && tid < head && blockIdx.y == 0) edge = tid;
        if (tid >= 8 && tid < 16 && blockIdx.y == splits - 1 && tail + tid - 8 < a.cols) edge = tail + tid - 8;
        const float edge_x = edge >= 0 ? Prec<DT>::to_f32(x[edge]) : -kInf;
        Given given = {false, 0.0f};
        if (tid == 0 && splits == 1) given = given_of<DT>(a, row);

        Part p = {kLowest, 0.0f, 0.0f};
        float most = -kInf;
        int at = -1;  // the piece with `most`
        uint4 raw[U];
        auto whole = [&](int v) { return P::raw((const elem_t*)__builtin_assume_aligned(base + (int64_t)v * VEC, 16)); };
        auto note = [&](float m, int v) {
            if (TOP && m > most) most = m, at = v;
        };
        int v = v0 + tid;
        if constexpr (HELD) {
            float m = -kInf;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * NT < v1) raw[u] = whole(v + u * NT);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * NT < v1) {
                    float f[VEC];
                    P::widen(raw[u], f);
                    const float mu = piece_max(f);
                    note(mu, v + u * NT);
                    m = fmaxf(m, mu);
                }
            p.m = fmaxf(p.m, m);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * NT < v1) {
                    float f[VEC];
                    P::widen(raw[u], f);
                    add_piece(p, f);
                }
        } else {
            for (; v + (U - 1) * NT < v1; v += U * NT) {
                float m[U];
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = whole(v + u * NT);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float f[VEC];
                    P::widen(raw[u], f);
                    m[u] = piece_max(f);
                    note(m[u], v + u * NT);
                }
                const float mm = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
                if (mm > p.m) rebase(p, mm);
                // (widened again: 32 floats kept from above would cost a third of the waves)
#pragma unroll
                for (int u = 0; u < U; ++u) asm volatile("" : "+v"(raw[u].x), "+v"(raw[u].y), "+v"(raw[u].z), "+v"(raw[u].w));
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float f[VEC];
                    P::widen(raw[u], f);
                    add_piece(p, f);
                }
            }
            for (; v < v1; v += NT) {
                float f[VEC];
                P::widen(whole(v), f);
                const float m = piece_max(f);
                note(m, v);
                if (m > p.m) rebase(p, m);
                add_piece(p, f);
            }
        }
        if (edge >= 0) {
            const float f[2] = {edge_x, -kInf};
            if (edge_x > p.m) rebase(p, edge_x);
            add_piece(p, f);
        }
        __syncthreads();  // the previous row's LDS is free
        // (made unknown here, or what the selection computes from it would be kept in registers while the row is read)
        int sel = threadIdx.x;
        asm volatile("" : "+v"(sel));
        const int lane = sel & 63, wave = sel >> 6;
        if constexpr (TOP) {
            if (at < 0 && v0 + sel < v1) at = v0 + sel;  // nothing but -inf
            maxima[sel] = at < 0 ? 0 : key_of(most, (uint32_t)at);
            for (int i = sel; i < kMostTop; i += NT) best[i] = 0;
            if (sel == 0) listed = 0, winners = 0;
        }
        p = block_join<W>(p, red);
        if constexpr (TOP) {
            if constexpr (W == 1) __syncthreads();
            if (wave == 0) {
                uint64_t k[2] = {maxima[lane], 0};
#pragma unroll
                for (int w = 1; w < W; ++w) k[w & 1] = maxima[w * 64 + lane] > k[w & 1] ? maxima[w * 64 + lane] : k[w & 1];
                const uint64_t b = bound_of_wave(k[0], k[1], a.top);
                if (lane == 0) bound = b;
            }
            __syncthreads();
            const uint64_t b = bound, mine = maxima[sel];
            const bool odd = !(p.s >= 0.0f);  // a NaN or an infinity
            // what is not below the bound in (value, piece) goes to the list
            const float b_value = b ? value_of((uint32_t)(b >> 32)) : -kInf;
            const uint32_t b_piece = b ? index_of(b) : 0xFFFFFFFFu;
            auto passes = [&](float f, int q) { return f > b_value || (f == b_value && (uint32_t)q <= b_piece); };
            if (!odd) {
                if (mine && mine >= b) winner[atomicAdd(&winners, 1)] = (uint16_t)sel;
                if (wave == 0) {
                    const bool in = edge >= 0 && passes(edge_x, edge < head ? 0 : whole_end);
                    if (__any(in)) {
                        const int to = take_room(in, &listed);
                        if (in && to < LIST) list[to] = key_of(edge_x, (uint32_t)edge);
                    }
                }
                __syncthreads();
                // the winners' pieces, `each` of them a winner, dealt to all threads, two at a time
                const int each = max(v1 - v0 + NT - 1, 0) / NT, all = winners * each;
                for (int i0 = 0; i0 < all; i0 += 2 * NT) {  // (all lanes: they count their entries together)
                    int q[2];
                    uint4 r[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int i = i0 + u * NT + sel, w = (int)((unsigned)i / (unsigned)each);
                        q[u] = i < all ? v0 + winner[w] + (i - w * each) * NT : v1;
                        if (q[u] < v1) r[u] = whole(q[u]);
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        float f[VEC];
                        uint32_t m = 0;
                        P::widen(r[u], f);
                        if (q[u] < v1) {
#pragma unroll
                            for (int e = 0; e < VEC; ++e) m |= (passes(f[e], q[u]) ? 1u : 0u) << e;
                        }
                        if (!__any(m != 0)) continue;
                        int to = take_room(__builtin_popcount(m), &listed);
#pragma unroll
                        for (int e = 0; e < VEC; ++e)
                            if ((m >> e) & 1) {
                                if (to < LIST) list[to] = key_of(f[e], (uint32_t)(q[u] * VEC - shift + e));
                                ++to;
                            }
                    }
                }
                __syncthreads();
            }
            if (!odd && listed <= LIST) {
                rank_keys<NT>(list, listed, best, a.top);
            } else {
                const int j0 = blockIdx.y == 0 ? 0 : min(v0 * VEC - shift, tail), j1 = blockIdx.y == splits - 1 ? a.cols : v1 * VEC - shift;
                uint64_t last = ~0ull;
                for (int i = 0; i < a.top; ++i) {
                    uint64_t k = 0;
                    for (int j = j0 + sel; j < j1; j += NT) {
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
                    if (sel == 0) best[i] = k;
                    last = k;
                }
            }
            __syncthreads();
        }
        if (splits == 1) {
            write_row<NT>(a, row, given, p, best);
        } else {
            char* ws = (char*)a.ws + (size_t)row * splits * part_bytes(a.top);
            if (sel == 0) ((float4*)ws)[blockIdx.y] = make_float4(p.m, p.s, p.sd, 0.0f);
            uint64_t* keys = (uint64_t*)(ws + 16 * (size_t)splits) + (size_t)blockIdx.y * a.top;
            for (int i = sel; i < a.top; i += NT) keys[i] = best[i];
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
    __shared__ uint64_t all[kMostSplits * kMostTop], list[kMostSplits * kMostTop], best[kMostTop], bound;
    __shared__ int listed;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t row = blockIdx.x;
    const char* ws = (const char*)a.ws + (size_t)row * splits * part_bytes(a.top);
    const uint64_t* keys = (const uint64_t*)(ws + 16 * (size_t)splits);
    const int n = splits * a.top;
    Given given = {false, 0.0f};
    if (tid == 0) given = given_of<DT>(a, row);
    // The lists are in order, so the first of each, or the first few where there are fewer than 128 lists, are the likeliest: their
    // top-th largest is the bound.  (Keys dealt to the lanes as they come put the firsts of 64 lists of 20 into 8 of 32 sets.)
    uint64_t first[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int o = tid + 64 * i;
        if (tid < 64 && o / splits < a.top) first[i] = keys[(o % splits) * a.top + o / splits];
    }
#pragma unroll 4
    for (int i = tid; i < n; i += NT) all[i] = keys[i];
    Part p = {kLowest, 0.0f, 0.0f};
    if (tid < splits) {
        const float4 f = ((const float4*)ws)[tid];
        p.m = f.x, p.s = f.y, p.sd = f.z;
    }
    if (tid == 0) listed = 0;
    for (int i = tid; i < kMostTop; i += NT) best[i] = 0;
    p = block_join<4>(p, red);
    if (a.top) {
        if (tid < 64) {
            const uint64_t b = bound_of_wave(first[0], first[1], a.top);
            if (lane == 0) bound = b ? b : 1;  // a key of 0 stands for no element
        }
        __syncthreads();
        const uint64_t b = bound;
        for (int i = tid; i - tid < n; i += NT) {
            const uint64_t k = i < n ? all[i] : 0;
            if (!__any(k >= b)) continue;
            const int to = take_room(k >= b, &listed);
            if (k >= b) list[to] = k;
        }
        __syncthreads();
        rank_keys<NT>(list, listed, best, a.top);
        __syncthreads();
    }
    write_row<NT>(a, row, given, p, best);
}

// The gradient: a piece of 16 bytes is read, and written, by one thread.  `per_row` threads (a power of two up to 256) share a row,
// or, for longer rows, a workgroup has 1024 pieces of one (`from`: such runs ahead of this launch's first).  x - lse = log p, so with c = g_logp + g_entropy (log p + entropy) every
// element is -p c, and the target's g_logp more.
template <int DT>
__global__ __launch_bounds__(256) void logprob_bwd_rows(LogprobArgs a, int per_row, int from)
{
    typedef typename Prec<DT>::elem_t elem_t;
    typedef Piece<DT> P;
    constexpr int VEC = P::VEC, U = 4;
    const int rows_here = 256 / per_row, l = threadIdx.x & (per_row - 1);
    const int pieces = (a.cols + VEC - 1) / VEC, first = (from + (int)blockIdx.y) * (per_row * U);
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
                f[k] = -p * __builtin_fmaf(gh, fmaxf(lp, -128.0f) + h, g);  // where p is 0, -inf and all below -88, the factor stays finite
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

// How a row is shared.  Waves a workgroup: one for rows of up to 256 pieces, which it holds; four up to 8192, so that several
// workgroups of a CU cover each other's selections; eight beyond (2048 rows, 5 alternatives, us with four / eight waves: 50257 bf16 53 / 61,
// 131072 bf16 110 / 104, 50257 fp32 81 / 79).  Fewer rows than CUs are shared by 256 / rows workgroups, as far as that leaves each of
// them two pieces a thread, up to 64 (256 rows of 50257 fp16 in one each 14 us, in two 17).  A row that starts within 16 bytes
// can touch a piece more than its length says: `pieces` is the most.  (More than 20 alternatives need the maxima of four waves.)
struct Shares {
    int waves, splits, share;
    bool held;
};
Shares shares_of(int64_t rows, int cols, int dtype, int top)
{
    const int vec = dtype == CONV_F32 ? 4 : 8, pieces = cols / vec + 2;
    Shares s;
    s.waves = pieces <= 256 ? 1 : pieces <= 8192 ? 4 : 8;
    int64_t want = pieces > 1024 ? (256 + rows - 1) / std::max<int64_t>(rows, 1) : 1;
    want = std::max<int64_t>(1, std::min<int64_t>({want, kMostSplits, pieces / 512}));
    if (want > 1 || (top > 20 && s.waves == 1)) s.waves = 4;
    s.share = (int)((pieces + want - 1) / want);
    s.splits = (pieces + s.share - 1) / s.share;
    s.held = s.share <= 4 * 64 * s.waves;
    return s;
}

template <int DT, int W, bool HELD>
void launch_w(const LogprobArgs& a, const Shares& sh, hipStream_t s)
{
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, 1 << 18), (unsigned)sh.splits), block(64 * W);
    if (a.top) hipLaunchKernelGGL((logprob_rows<DT, W, HELD, true>), grid, block, 0, s, a, sh.splits, sh.share);
    else hipLaunchKernelGGL((logprob_rows<DT, W, HELD, false>), grid, block, 0, s, a, sh.splits, sh.share);
}

template <int DT>
hipError_t fwd(const LogprobArgs& a, hipStream_t s)
{
    const Shares sh = shares_of(a.rows, a.cols, DT, a.top);
    if (sh.waves == 1) launch_w<DT, 1, true>(a, sh, s);
    else if (sh.waves == 4 && sh.held) launch_w<DT, 4, true>(a, sh, s);
    else if (sh.waves == 4) launch_w<DT, 4, false>(a, sh, s);
    else launch_w<DT, 8, false>(a, sh, s);
    if (sh.splits > 1) hipLaunchKernelGGL((logprob_join<DT>), dim3((unsigned)a.rows), dim3(256), 0, s, a, sh.splits);
    return hipGetLastError();
}

}  // namespace

size_t logprob_workspace(int64_t rows, int cols, int top, int dtype)
{
    const Shares sh = shares_of(rows, cols, dtype, top);
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
    const int runs = (pieces + per_row * 4 - 1) / (per_row * 4);
    // gridDim.y is at most 65535: rows of more than 65535 x 1024 pieces (fp32 from 268 million columns) take several launches
    for (int from = 0; from < runs; from += 65535) {
        const dim3 grid((unsigned)std::min<int64_t>(blocks, 1 << 20), (unsigned)std::min(runs - from, 65535));
        hipLaunchKernelGGL((logprob_bwd_rows<DT>), grid, dim3(256), 0, s, a, per_row, from);
    }
    return hipGetLastError();
}

hipError_t launch_logprob_bwd(LogprobArgs& a, int dtype, hipStream_t s)
{
    return dtype == CONV_F32 ? bwd<CONV_F32>(a, s) : dtype == CONV_F16 ? bwd<CONV_F16>(a, s) : bwd<CONV_BF16>(a, s);
}

}  // namespace convfwd
