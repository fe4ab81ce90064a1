// What stands between two blocks of rows, in one pass forward and one backward:
//
//   u = norm(h) gamma_h + beta_h  (or h),   r_out = r + scale gate u,   y = norm(r_out before it is rounded) gamma + beta
//
// The rows are held in registers as in layer norm: G neighbouring lanes share a row, each with up to 16 of its elements (backward 8: with 16 there were 256 registers,
// spilled ones and two waves a SIMD), forward a workgroup of as many waves as the row takes (G = 0).  scale is folded into gamma_h and beta_h, so a lane keeps four vectors of its columns forward, three
// backward.  Backward, with q the gradient at the sum,
//
//   q = dr_out + rstd (dy gamma - avg - xh avg),   dr = q,   dh = rstd_h (g - avg g - hh avg(g hh)),  g = q gate scale gamma_h,
//   dgamma = sum dy xh,  dbeta = sum dy,  and from S1 = sum p and S2 = sum p hh over the rows, p = q gate:
//   dgamma_h = scale S2,  dbeta_h = scale S1,  dscale = gamma_h S2 + beta_h S1.
//
// Where rows share a gate, the sums S1 and S2 are formed for each gate row apart, without the gate: its gradient is scale (gamma_h S2 + beta_h S1)
// then, and the sums over all rows are those times the gate.  A workgroup takes `items`: runs of rows, each within one gate row; a lane
// adds up its columns in registers, a workgroup's lanes meet in LDS, and a second kernel adds the items, always in the same order.
// Bound by memory: four tensors forward (50176 x 768 bf16 with shared gates 76 us, 4.1 TB/s), six backward and with gates of their own eight (16384 x 4096 bf16 221 us,
// 4.9 TB/s); few rows by two launches (3380 x 384 fp32 backward 11.2 us and 7.2 for the join).
#pragma once

#include <algorithm>

#include "held_rows.h"

namespace convfwd {

// Runs of rows that a workgroup adds up apart: `per` runs of `each` rows in every stretch of `stretch` rows (a gate's, or all).
__device__ __forceinline__ void item_rows(const ResidualNormArgs& a, int64_t item, int64_t& first, int64_t& last)
{
    const int64_t g = item / a.per, part = item - g * a.per;
    first = g * a.stretch + part * a.each;
    last = min(min(first + a.each, (g + 1) * a.stretch), a.rows);
}

__device__ __forceinline__ float gate_of(float g, int sigmoid) { return sigmoid ? __builtin_amdgcn_rcpf(1.0f + __expf(-g)) : g; }

// A gate of each row's own, or one that rows share.
enum { NO_GATE = 0, OWN_GATE = 1, SHARED_GATE = 2 };

// PLAIN calls have all tensors and rows of whole pieces: without a branch for each tensor and a mask for each element the backward
// kernel takes half the instructions, which bound it.  A lane's piece is then in the row or behind it.
template <int N>
__device__ __forceinline__ void keep_if(bool live, uint4 (&raw)[N], int i)
{
    raw[i].x = live ? raw[i].x : 0, raw[i].y = live ? raw[i].y : 0, raw[i].z = live ? raw[i].z : 0, raw[i].w = live ? raw[i].w : 0;
}

template <int DT, int G, int NV, int MAXT, bool POST, int GATE, bool PLAIN>
__global__ __launch_bounds__(MAXT) void residual_norm_fwd_rows(ResidualNormArgs a)
{
    typedef Held<DT, G, NV> H;
    typedef typename H::elem_t elem_t;
    constexpr int VEC = H::VEC, ROWS = G ? MAXT / G : 1;
    __shared__ float red[4][G ? 1 : 16];
    const int l = G ? threadIdx.x % G : threadIdx.x;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + (G ? threadIdx.x / G : 0);
    const float inv_cols = 1.0f / (float)a.cols;
    uint4 nr[NV], nh[NV], ng[NV];
    auto load = [&](int64_t t) {
        t = t < a.rows ? t : a.rows - 1;
        H::load(nr, (const elem_t*)a.r + t * a.ldr, a.cols, l);
        H::load(nh, (const elem_t*)a.h + t * a.ldh, a.cols, l);
        if constexpr (GATE != NO_GATE) H::load(ng, (const elem_t*)a.gate + (int64_t)((uint32_t)t / (uint32_t)a.gate_rows) * a.ldg, a.cols, l);
    };
    constexpr bool AHEAD = NV * VEC < 16 || DT != CONV_F32;
    if (AHEAD) load(row);
    float ga[NV][VEC], gb[NV][VEC], gamma[NV][VEC], beta[NV][VEC];
    {
        H::columns(gb, a.scale, 1.0f, a.cols, l);
        if constexpr (POST) {
            H::columns(ga, a.gamma_h, 1.0f, a.cols, l);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) ga[i][k] *= gb[i][k];
            float b[NV][VEC];
            H::columns(b, a.beta_h, 0.0f, a.cols, l);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) gb[i][k] *= b[i][k];
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) ga[i][k] = gb[i][k];
        }
        H::columns(gamma, a.gamma, 1.0f, a.cols, l);
        H::columns(beta, a.beta, 0.0f, a.cols, l);
    }
    bool live[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) live[i] = (i * H::lanes() + l) * VEC < a.cols;
    auto clear = [&](uint4 (&raw)[NV]) {
        if constexpr (PLAIN) {
#pragma unroll
            for (int i = 0; i < NV; ++i) keep_if(live[i], raw, i);
        } else {
            H::clear(raw, a.cols, l);
        }
    };
    auto store = [&](elem_t* to, const float (&v)[VEC], int i) {
        if constexpr (PLAIN) {
            if (live[i]) H::P::put(to + (i * H::lanes() + l) * VEC, H::P::narrow(v));
        } else {
            H::store(to, v, a.cols, i, l);
        }
    };
    // the statistics of held values, which are left centred
    auto normed = [&](float (&x)[NV][VEC], int at, float& mean, float& rstd) {
        mean = 0.0f;
        if (!a.rms) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) sum += x[i][k];
            mean = row_reduce<G, OpSum>(sum, red[at]) * inv_cols;
        }
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int left = a.cols - (i * H::lanes() + l) * VEC;
            const float m = !PLAIN || live[i] ? mean : 0.0f;
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                x[i][k] -= m;
                if (!PLAIN && left < VEC) x[i][k] = k < left ? x[i][k] : 0.0f;
                sq = __builtin_fmaf(x[i][k], x[i][k], sq);
            }
        }
        rstd = 1.0f / sqrtf(row_reduce<G, OpSum>(sq, red[at + 1]) * inv_cols + a.eps);
    };
    // every lane of a workgroup makes the same number of rounds: the reductions of wide rows have barriers
    for (int64_t first = (int64_t)blockIdx.x * ROWS; first < a.rows; first += step, row += step) {
        if (!AHEAD) load(row);
        float x[NV][VEC], u[NV][VEC], g[NV][VEC];
        clear(nr);
        clear(nh);
        if constexpr (GATE != NO_GATE) clear(ng);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            H::P::widen(nr[i], x[i]);
            H::P::widen(nh[i], u[i]);
            if constexpr (GATE != NO_GATE) H::P::widen(ng[i], g[i]);
        }
        if (AHEAD && first + step < a.rows) load(row + step);
        float mean_h = 0.0f, rstd_h = 1.0f, mean = 0.0f, rstd = 1.0f;
        if constexpr (POST) normed(u, 0, mean_h, rstd_h);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                float v = POST ? __builtin_fmaf(u[i][k] * rstd_h, ga[i][k], gb[i][k]) : u[i][k] * ga[i][k];
                if constexpr (GATE != NO_GATE) v *= gate_of(g[i][k], a.sigmoid);
                x[i][k] += v;
            }
        const bool in = row < a.rows;
        // r_out may be r: every wave has read its pieces before any is written (a row's last piece is read across two waves' columns)
        if constexpr (G == 0) {
            if (!POST) __syncthreads();
        }
        if (in) {
#pragma unroll
            for (int i = 0; i < NV; ++i) store((elem_t*)a.r_out + row * a.ldr, x[i], i);
        }
        if (PLAIN || a.y) {
            // (past the row's end there may be beta_h's zeros only)
            normed(x, 2, mean, rstd);
            if (in) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) x[i][k] = __builtin_fmaf(x[i][k] * rstd, gamma[i][k], beta[i][k]);
                    store((elem_t*)a.y + row * a.ldy, x[i], i);
                }
            }
        }
        if (in && l == 0 && (PLAIN || a.stats_out)) *(float4*)(a.stats_out + row * 4) = make_float4(mean_h, rstd_h, mean, rstd);
        if constexpr (G == 0) __syncthreads();  // the next row's reductions use the same LDS
    }
}

// Sums of `x` and `y` over the sets of lanes with the same columns, to set 0.
template <int G, int N, int SETS>
__device__ __forceinline__ void sets_sum(float (&x)[N], float (&y)[N], float* lds, int set, bool holder, int l)
{
    if constexpr (G < 64) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = across_rows<G>(x[k]), y[k] = across_rows<G>(y[k]);
    }
#pragma unroll
    for (int half = SETS / 2; half >= 1; half /= 2) {
        float* p = lds + (set % half) * (2 * G * N) + l;  // a lane's neighbours are next to it: no bank twice
        if (set >= half && set < 2 * half && holder) {
#pragma unroll
            for (int k = 0; k < N; ++k) p[k * G] = x[k], p[(N + k) * G] = y[k];
        }
        __syncthreads();
        if (set < half && holder) {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] += p[k * G], y[k] += p[(N + k) * G];
        }
        __syncthreads();
    }
}

// Where a lane holds 16 elements (a workgroup of 1024 a row) there are no registers for the column sums: it leaves the averages of each
// row, and residual_norm_sums reads the tensors again.
// (Registers for three workgroups of 256 a CU, or one of 512 or 1024.)
template <int DT, int G, int NV, int NT, bool POST, int GATE, bool PLAIN>
__global__ __launch_bounds__(NT, NT == 256 ? 3 : 1) void residual_norm_bwd_rows(ResidualNormArgs a)
{
    typedef Held<DT, G, NV> H;
    typedef typename H::elem_t elem_t;
    constexpr int VEC = H::VEC, N = NV * VEC, ROWS = NT / G, WAVES = NT / 64, SETS = G <= 64 ? WAVES : ROWS;
    constexpr bool SUMS = N <= 8;
    __shared__ float red[2][WAVES];
    __shared__ float lds[SUMS && SETS > 1 ? SETS / 2 * 2 * G * N : 1];
    const int tid = threadIdx.x, l = tid % G;
    const float inv_cols = 1.0f / (float)a.cols;
    const int set = G <= 64 ? tid / 64 : tid / G;
    const bool holder = G >= 64 || (tid & 63) < G;

    auto reduce2 = [&](float& s1, float& s2) {
        if constexpr (G <= 64) {
            s1 = lanes_reduce<G, OpSum>(s1), s2 = lanes_reduce<G, OpSum>(s2);
        } else {
            // the waves of this row; other rows of the workgroup have waves of their own
            constexpr int W = G / 64;
            s1 = lanes_reduce<64, OpSum>(s1), s2 = lanes_reduce<64, OpSum>(s2);
            const int wave = tid >> 6, w0 = wave / W * W;
            if ((tid & 63) == 0) red[0][wave] = s1, red[1][wave] = s2;
            __syncthreads();
            s1 = lanes_reduce<W, OpSum>(red[0][w0 + (tid & (W - 1))]), s2 = lanes_reduce<W, OpSum>(red[1][w0 + (tid & (W - 1))]);
            __syncthreads();
        }
        s1 = a.rms ? 0.0f : s1 * inv_cols, s2 *= inv_cols;
    };
    auto flush = [&](float* to, float (&x)[NV][VEC], float (&y)[NV][VEC]) {
        float fx[N], fy[N];
        __builtin_memcpy(fx, x, sizeof(fx));
        __builtin_memcpy(fy, y, sizeof(fy));
        sets_sum<G, N, SETS>(fx, fy, lds, set, holder, l);
        if (set == 0 && holder) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = (i * G + l) * VEC;
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    if (j + k < a.cols) to[j + k] = fx[i * VEC + k], to[a.cols + j + k] = fy[i * VEC + k];
            }
        }
    };

    float gamma[NV][VEC], ga[NV][VEC], gb[NV][VEC];
    auto vectors_of_y = [&]() { H::columns(gamma, a.gamma, 1.0f, a.cols, l); };
    auto vectors_of_h = [&]() {
        H::columns(gb, a.scale, 1.0f, a.cols, l);
        if constexpr (POST) {
            H::columns(ga, a.gamma_h, 1.0f, a.cols, l);
            float b[NV][VEC];
            H::columns(b, a.beta_h, 0.0f, a.cols, l);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) ga[i][k] *= gb[i][k], gb[i][k] *= b[i][k];
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) ga[i][k] = gb[i][k], gb[i][k] = 0.0f;
        }
    };
    if constexpr (SUMS) vectors_of_y(), vectors_of_h();
    float dg[NV][VEC], db[NV][VEC], s1[NV][VEC], s2[NV][VEC];
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < VEC; ++k) dg[i][k] = db[i][k] = s1[i][k] = s2[i][k] = 0.0f;
    }

    const bool has_dy = PLAIN || a.dy, has_dr_out = PLAIN || a.dr_out;
    bool live[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) live[i] = (i * G + l) * VEC < a.cols;
    auto clear = [&](uint4 (&raw)[NV]) {
        if constexpr (PLAIN) {
#pragma unroll
            for (int i = 0; i < NV; ++i) keep_if(live[i], raw, i);
        } else {
            H::clear(raw, a.cols, l);
        }
    };
    auto store = [&](elem_t* to, const float (&v)[VEC], int i) {
        if constexpr (PLAIN) {
            if (live[i]) H::P::put(to + (i * G + l) * VEC, H::P::narrow(v));
        } else {
            H::store(to, v, a.cols, i, l);
        }
    };
    // The tensors of a row are asked for a round ahead, each as soon as the present one's is taken apart, where they are 16 bits (the same registers).
    constexpr bool AHEAD = DT != CONV_F32 && SUMS;
    uint4 nx[NV], ndy[NV], nh[NV], ndr[NV], ng[NV];
    float4 nst;
    auto load_y = [&](int64_t t) {
        if (has_dy) {
            H::load(nx, (const elem_t*)a.x + t * a.ldr, a.cols, l);
            H::load(ndy, (const elem_t*)a.dy + t * a.ldy, a.cols, l);
        }
        nst = PLAIN || a.stats ? *(const float4*)(a.stats + t * 4) : make_float4(0.0f, 1.0f, 0.0f, 1.0f);
    };
    auto load_dr = [&](int64_t t) {
        if (has_dr_out) H::load(ndr, (const elem_t*)a.dr_out + t * a.ldr, a.cols, l);
    };
    auto load_h = [&](int64_t t) {
        H::load(nh, (const elem_t*)a.h + t * a.ldh, a.cols, l);
        if constexpr (GATE != NO_GATE) H::load(ng, (const elem_t*)a.gate + (int64_t)((uint32_t)t / (uint32_t)a.gate_rows) * a.ldg, a.cols, l);
    };
    auto row_of = [&](int64_t at, int64_t end) { return min(at + tid / G, end - 1); };
    int64_t item = blockIdx.x, begin, end;
    if (item < a.items) {
        item_rows(a, item, begin, end);
        if constexpr (AHEAD) load_y(row_of(begin, end)), load_dr(row_of(begin, end)), load_h(row_of(begin, end));
    }
    while (item < a.items) {
        const int64_t next_item = item + gridDim.x;
        int64_t next_begin = 0, next_end = 0;
        if (next_item < a.items) item_rows(a, next_item, next_begin, next_end);
        for (int64_t at = begin; at < end; at += ROWS) {
            const int64_t row = at + tid / G;
            const bool in = row < end;
            const int64_t t = in ? row : end - 1;
            // (behind the last round of all the same row again)
            const int64_t ahead = at + ROWS < end ? row_of(at + ROWS, end) : next_item < a.items ? row_of(next_begin, next_end) : t;
            if constexpr (!AHEAD) load_y(t);
            constexpr bool EARLY = G < 512;  // (where there are registers for all of a row's tensors)
            if constexpr (!AHEAD && EARLY) load_dr(t), load_h(t);
            const float4 st = nst;
            float q[NV][VEC];
            float c1 = 0.0f, c2 = 0.0f;
            if (has_dy) {
                if constexpr (!SUMS) vectors_of_y();
                float x[NV][VEC];
                if constexpr (!PLAIN) H::clear(nx, a.cols, l);
                clear(ndy);
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    H::P::widen(nx[i], x[i]);
                    H::P::widen(ndy[i], q[i]);
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        x[i][k] = (x[i][k] - st.z) * st.w;  // past the end dy is 0
                        if constexpr (SUMS) {
                            if (in) {
                                dg[i][k] = __builtin_fmaf(q[i][k], x[i][k], dg[i][k]);
                                db[i][k] += q[i][k];
                            }
                        }
                        q[i][k] *= gamma[i][k];
                        c1 += q[i][k];
                        c2 = __builtin_fmaf(q[i][k], x[i][k], c2);
                    }
                }
                if constexpr (AHEAD) load_y(ahead);
                reduce2(c1, c2);
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int left = a.cols - (i * G + l) * VEC;
                    const float rstd = !PLAIN || live[i] ? st.w : 0.0f;
#pragma unroll
                    for (int k = 0; k < VEC; ++k) {
                        q[i][k] = rstd * (q[i][k] - c1 - x[i][k] * c2);
                        if (!PLAIN && left < VEC) q[i][k] = k < left ? q[i][k] : 0.0f;
                    }
                }
            } else {
                if constexpr (AHEAD) load_y(ahead);
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) q[i][k] = 0.0f;
            }
            if constexpr (!AHEAD && !EARLY) load_dr(t), load_h(t);
            if constexpr (!SUMS) {
                if (in && l == 0) a.averages[row * 2] = c1, a.averages[row * 2 + 1] = c2;
            }
            if (has_dr_out) {
                clear(ndr);
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float d[VEC];
                    H::P::widen(ndr[i], d);
#pragma unroll
                    for (int k = 0; k < VEC; ++k) q[i][k] += d[k];
                }
                if constexpr (AHEAD) load_dr(ahead);
            }
            if (in && (PLAIN || a.dr)) {
#pragma unroll
                for (int i = 0; i < NV; ++i) store((elem_t*)a.dr + row * a.ldr, q[i], i);
            }
            if constexpr (!SUMS) vectors_of_h();
            float hh[NV][VEC], gates[NV][VEC];
            if constexpr (!PLAIN) {
                H::clear(nh, a.cols, l);
                if constexpr (GATE != NO_GATE) H::clear(ng, a.cols, l);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                H::P::widen(nh[i], hh[i]);
                if constexpr (GATE != NO_GATE) H::P::widen(ng[i], gates[i]);
            }
            if constexpr (AHEAD) load_h(ahead);
            float d1 = 0.0f, d2 = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const float(&g)[VEC] = gates[i];
                float dgate[VEC];
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    if constexpr (POST) hh[i][k] = (hh[i][k] - st.x) * st.y;
                    float p = q[i][k], sum = p;
                    if constexpr (GATE != NO_GATE) {
                        const float gate = gate_of(g[k], a.sigmoid);
                        if constexpr (GATE == OWN_GATE) {
                            dgate[k] = p * (POST ? __builtin_fmaf(hh[i][k], ga[i][k], gb[i][k]) : hh[i][k] * ga[i][k]);
                            if (a.sigmoid) dgate[k] *= gate * (1.0f - gate);
                        }
                        p *= gate;
                        if constexpr (GATE == OWN_GATE) sum = p;
                    }
                    if constexpr (SUMS) {
                        if (in) {
                            s1[i][k] += sum;
                            s2[i][k] = __builtin_fmaf(sum, hh[i][k], s2[i][k]);
                        }
                    }
                    q[i][k] = p * ga[i][k];
                    if constexpr (POST) {
                        d1 += q[i][k];
                        d2 = __builtin_fmaf(q[i][k], hh[i][k], d2);
                    }
                }
                if (GATE == OWN_GATE && in && (PLAIN || a.dgate)) store((elem_t*)a.dgate + row * a.ldg, dgate, i);
            }
            if (PLAIN || a.dh) {
                if constexpr (POST) reduce2(d1, d2);
                if (in) {
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        if constexpr (POST) {
#pragma unroll
                            for (int k = 0; k < VEC; ++k) q[i][k] = st.y * (q[i][k] - d1 - hh[i][k] * d2);
                        }
                        store((elem_t*)a.dh + row * a.ldh, q[i], i);
                    }
                }
            }
        }
        if constexpr (SUMS) {
            if (a.sums_h) {
                flush(a.sums_h + item * 2 * a.cols, s1, s2);
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) s1[i][k] = s2[i][k] = 0.0f;
            }
        }
        item = next_item, begin = next_begin, end = next_end;
    }
    if constexpr (SUMS) {
        if (a.sums) flush(a.sums + (int64_t)blockIdx.x * 2 * a.cols, dg, db);
    }
}

template <int DT, int G, int NV, bool POST, int GATE, bool PLAIN>
void residual_norm_fwd_launch(const ResidualNormArgs& a, int waves, hipStream_t s)
{
    constexpr int CUS = 256;
    const int rows = G ? 256 / G : 1;
    const int64_t blocks = std::min<int64_t>((a.rows + rows - 1) / rows, CUS * std::max(1, 16 / waves));
    if (G) hipLaunchKernelGGL((residual_norm_fwd_rows<DT, G, NV, 256, POST, GATE, PLAIN>), dim3((unsigned)blocks), dim3(256), 0, s, a);
    else if constexpr (G == 0) {
        if (waves <= 8) hipLaunchKernelGGL((residual_norm_fwd_rows<DT, 0, NV, 512, POST, GATE, PLAIN>), dim3((unsigned)blocks), dim3(64 * waves), 0, s, a);
        else hipLaunchKernelGGL((residual_norm_fwd_rows<DT, 0, NV, 1024, POST, GATE, PLAIN>), dim3((unsigned)blocks), dim3(64 * waves), 0, s, a);
    }
}

// `most` elements a lane: 8 or 16, and one piece of fp32 in rows of eight lanes (Held loads rows shorter than a piece only there)
template <int DT, int G, bool POST, int GATE, bool PLAIN>
void residual_norm_fwd_pieces(const ResidualNormArgs& a, int most, int waves, hipStream_t s)
{
    constexpr int VEC = DT == CONV_F32 ? 4 : 8;
    if constexpr (G == 8 && VEC == 4) {
        if (most == 4) return residual_norm_fwd_launch<DT, G, 1, POST, GATE, PLAIN>(a, waves, s);
    }
    if (most == 8) residual_norm_fwd_launch<DT, G, 8 / VEC, POST, GATE, PLAIN>(a, waves, s);
    else residual_norm_fwd_launch<DT, G, 16 / VEC, POST, GATE, PLAIN>(a, waves, s);
}

struct FwdHeld {
    static constexpr bool GATES_ALIKE = true;
    template <int DT, bool POST, int GATE, bool PLAIN>
    static void run(const ResidualNormArgs& a, const ResidualNormForm& f, hipStream_t s)
    {
        if (f.lanes == 8) residual_norm_fwd_pieces<DT, 8, POST, GATE, PLAIN>(a, f.most, 4, s);
        else if (f.lanes == 16) residual_norm_fwd_pieces<DT, 16, POST, GATE, PLAIN>(a, f.most, 4, s);
        else if (f.lanes == 64) residual_norm_fwd_pieces<DT, 64, POST, GATE, PLAIN>(a, f.most, 4, s);
        else residual_norm_fwd_pieces<DT, 0, POST, GATE, PLAIN>(a, f.most, f.waves, s);
    }
};

struct BwdHeld {
    static constexpr bool GATES_ALIKE = false;
    template <int DT, int G, int NV, int NT, bool POST, int GATE, bool PLAIN>
    static void launch(const ResidualNormArgs& a, const ResidualNormForm& f, hipStream_t s)
    {
        hipLaunchKernelGGL((residual_norm_bwd_rows<DT, G, NV, NT, POST, GATE, PLAIN>), dim3((unsigned)f.groups), dim3(NT), 0, s, a);
    }
    template <int DT, bool POST, int GATE, bool PLAIN>
    static void run(const ResidualNormArgs& a, const ResidualNormForm& f, hipStream_t s)
    {
        constexpr int VEC = DT == CONV_F32 ? 4 : 8;
        if constexpr (VEC == 4) {
            if (f.most == 4) return launch<DT, 8, 1, 256, POST, GATE, PLAIN>(a, f, s);
        }
        switch (f.lanes) {
            case 8: return launch<DT, 8, 8 / VEC, 256, POST, GATE, PLAIN>(a, f, s);
            case 16: return launch<DT, 16, 8 / VEC, 256, POST, GATE, PLAIN>(a, f, s);
            case 32: return launch<DT, 32, 8 / VEC, 256, POST, GATE, PLAIN>(a, f, s);
            case 64: return launch<DT, 64, 8 / VEC, 256, POST, GATE, PLAIN>(a, f, s);
            case 128: return launch<DT, 128, 8 / VEC, 256, POST, GATE, PLAIN>(a, f, s);
            case 256: return launch<DT, 256, 8 / VEC, 256, POST, GATE, PLAIN>(a, f, s);
            case 512: return launch<DT, 512, 8 / VEC, 512, POST, GATE, PLAIN>(a, f, s);
            default:
                if (f.most == 8) return launch<DT, 1024, 8 / VEC, 1024, POST, GATE, PLAIN>(a, f, s);
                return launch<DT, 1024, 16 / VEC, 1024, POST, GATE, PLAIN>(a, f, s);
        }
    }
};

template <int DT, typename F>
hipError_t residual_norm_held(const ResidualNormArgs& a, const ResidualNormForm& f, bool all, hipStream_t s)
{
    const bool plain = all && a.cols % (DT == CONV_F32 ? 4 : 8) == 0;
    const int gate = !a.gate ? NO_GATE : a.gate_rows == 1 || F::GATES_ALIKE ? OWN_GATE : SHARED_GATE;
#define CONVFWD_WITH(POST, GATE) \
    if ((a.post != 0) == POST && gate == GATE) plain ? F::template run<DT, POST, GATE, true>(a, f, s) : F::template run<DT, POST, GATE, false>(a, f, s);
    CONVFWD_WITH(true, NO_GATE)
    CONVFWD_WITH(true, OWN_GATE)
    CONVFWD_WITH(false, NO_GATE)
    CONVFWD_WITH(false, OWN_GATE)
    if constexpr (!F::GATES_ALIKE) {
        CONVFWD_WITH(true, SHARED_GATE)
        CONVFWD_WITH(false, SHARED_GATE)
    }
#undef CONVFWD_WITH
    return hipGetLastError();
}
template <int DT>
hipError_t residual_norm_fwd_held(const ResidualNormArgs& a, const ResidualNormForm& f, hipStream_t s)
{
    return residual_norm_held<DT, FwdHeld>(a, f, a.y && a.stats_out, s);
}
template <int DT>
hipError_t residual_norm_bwd_held(const ResidualNormArgs& a, const ResidualNormForm& f, hipStream_t s)
{
    const bool all = a.dy && a.dr_out && a.dr && a.dh && a.stats && (!a.gate || a.gate_rows > 1 || a.dgate);
    return residual_norm_held<DT, BwdHeld>(a, f, all, s);
}

}  // namespace convfwd
