// The norms around a block: which form a call takes, rows that no registers hold, and the joins of the backward pass.
#include "residual_norm_kernel.h"

namespace convfwd {

namespace {

constexpr int kCUs = 256;

// ---- rows of any length: a workgroup a row, an element a load, the row read again for every pass ---------------------------------

template <int DT>
__global__ __launch_bounds__(1024) void residual_norm_fwd_any(ResidualNormArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    constexpr int NT = 1024;
    __shared__ float red[4][16];
    for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const elem_t *r = (const elem_t*)a.r + t * a.ldr, *h = (const elem_t*)a.h + t * a.ldh;
        const elem_t* gate = a.gate ? (const elem_t*)a.gate + t / a.gate_rows * a.ldg : nullptr;
        float mean_h = 0.0f, rstd_h = 1.0f, mean = 0.0f, rstd = 1.0f;
        if (a.post) {
            float sum = 0.0f, sq = 0.0f;
            if (!a.rms) {
                for (int j = threadIdx.x; j < a.cols; j += NT) sum += Prec<DT>::to_f32(h[j]);
                mean_h = block_reduce<16, OpSum>(sum, red[0]) / (float)a.cols;
            }
            for (int j = threadIdx.x; j < a.cols; j += NT) {
                const float d = Prec<DT>::to_f32(h[j]) - mean_h;
                sq = __builtin_fmaf(d, d, sq);
            }
            rstd_h = 1.0f / sqrtf(block_reduce<16, OpSum>(sq, red[1]) / (float)a.cols + a.eps);
        }
        auto sum_at = [&](int j) {
            float v = Prec<DT>::to_f32(h[j]), s = a.scale ? a.scale[j] : 1.0f;
            if (a.post) v = __builtin_fmaf((v - mean_h) * rstd_h, s * (a.gamma_h ? a.gamma_h[j] : 1.0f), s * (a.beta_h ? a.beta_h[j] : 0.0f));
            else v *= s;
            if (gate) v *= gate_of(Prec<DT>::to_f32(gate[j]), a.sigmoid);
            return Prec<DT>::to_f32(r[j]) + v;
        };
        if (a.y) {
            float sum = 0.0f, sq = 0.0f;
            if (!a.rms) {
                for (int j = threadIdx.x; j < a.cols; j += NT) sum += sum_at(j);
                mean = block_reduce<16, OpSum>(sum, red[2]) / (float)a.cols;
            }
            for (int j = threadIdx.x; j < a.cols; j += NT) {
                const float d = sum_at(j) - mean;
                sq = __builtin_fmaf(d, d, sq);
            }
            rstd = 1.0f / sqrtf(block_reduce<16, OpSum>(sq, red[3]) / (float)a.cols + a.eps);
        }
        for (int j = threadIdx.x; j < a.cols; j += NT) {
            const float x = sum_at(j);
            ((elem_t*)a.r_out)[t * a.ldr + j] = Prec<DT>::from_f32(x);
            if (a.y)
                ((elem_t*)a.y)[t * a.ldy + j] = Prec<DT>::from_f32(__builtin_fmaf((x - mean) * rstd, a.gamma ? a.gamma[j] : 1.0f, a.beta ? a.beta[j] : 0.0f));
        }
        if (threadIdx.x == 0 && a.stats_out) *(float4*)(a.stats_out + t * 4) = make_float4(mean_h, rstd_h, mean, rstd);
        __syncthreads();
    }
}

// The gradient at the sum at one element; c1, c2: the averages of the row that the norm's gradient takes away.
template <int DT>
__device__ __forceinline__ float grad_at(const ResidualNormArgs& a, int64_t t, int j, float4 st, float c1, float c2)
{
    typedef typename Prec<DT>::elem_t elem_t;
    float q = a.dr_out ? Prec<DT>::to_f32(((const elem_t*)a.dr_out)[t * a.ldr + j]) : 0.0f;
    if (a.dy) {
        const float xh = (Prec<DT>::to_f32(((const elem_t*)a.x)[t * a.ldr + j]) - st.z) * st.w;
        const float g = Prec<DT>::to_f32(((const elem_t*)a.dy)[t * a.ldy + j]) * (a.gamma ? a.gamma[j] : 1.0f);
        q += st.w * (g - c1 - xh * c2);
    }
    return q;
}
__device__ __forceinline__ float4 stats_of(const ResidualNormArgs& a, int64_t t)
{
    return a.stats ? *(const float4*)(a.stats + t * 4) : make_float4(0.0f, 1.0f, 0.0f, 1.0f);
}

// dr, dh and the gradients of gates of a row's own; leaves the averages of each row for the column sums.
template <int DT>
__global__ __launch_bounds__(1024) void residual_norm_bwd_any(ResidualNormArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    constexpr int NT = 1024;
    __shared__ float red[4][16];
    const float inv_cols = 1.0f / (float)a.cols;
    for (int64_t t = blockIdx.x; t < a.rows; t += gridDim.x) {
        const float4 st = stats_of(a, t);
        const elem_t* h = (const elem_t*)a.h + t * a.ldh;
        const elem_t* gate = a.gate ? (const elem_t*)a.gate + t / a.gate_rows * a.ldg : nullptr;
        float c1 = 0.0f, c2 = 0.0f, d1 = 0.0f, d2 = 0.0f;
        if (a.dy) {
            for (int j = threadIdx.x; j < a.cols; j += NT) {
                const float xh = (Prec<DT>::to_f32(((const elem_t*)a.x)[t * a.ldr + j]) - st.z) * st.w;
                const float g = Prec<DT>::to_f32(((const elem_t*)a.dy)[t * a.ldy + j]) * (a.gamma ? a.gamma[j] : 1.0f);
                c1 += g, c2 = __builtin_fmaf(g, xh, c2);
            }
            c1 = block_reduce<16, OpSum>(c1, red[0]), c2 = block_reduce<16, OpSum>(c2, red[1]) * inv_cols;
            c1 = a.rms ? 0.0f : c1 * inv_cols;
        }
        auto at_hh = [&](int j, float q, float gv) {  // the gradient at the normed h
            const float s = a.scale ? a.scale[j] : 1.0f;
            return q * gv * (a.post && a.gamma_h ? s * a.gamma_h[j] : s);
        };
        if (a.post && a.dh) {
            for (int j = threadIdx.x; j < a.cols; j += NT) {
                const float g = at_hh(j, grad_at<DT>(a, t, j, st, c1, c2), gate ? gate_of(Prec<DT>::to_f32(gate[j]), a.sigmoid) : 1.0f);
                d1 += g, d2 = __builtin_fmaf(g, (Prec<DT>::to_f32(h[j]) - st.x) * st.y, d2);
            }
            d1 = block_reduce<16, OpSum>(d1, red[2]), d2 = block_reduce<16, OpSum>(d2, red[3]) * inv_cols;
            d1 = a.rms ? 0.0f : d1 * inv_cols;
        }
        for (int j = threadIdx.x; j < a.cols; j += NT) {
            const float q = grad_at<DT>(a, t, j, st, c1, c2), gv = gate ? gate_of(Prec<DT>::to_f32(gate[j]), a.sigmoid) : 1.0f;
            const float hh = a.post ? (Prec<DT>::to_f32(h[j]) - st.x) * st.y : Prec<DT>::to_f32(h[j]);
            if (a.dr) ((elem_t*)a.dr)[t * a.ldr + j] = Prec<DT>::from_f32(q);
            if (a.dh) {
                const float g = at_hh(j, q, gv);
                ((elem_t*)a.dh)[t * a.ldh + j] = Prec<DT>::from_f32(a.post ? st.y * (g - d1 - hh * d2) : g);
            }
            if (gate && a.gate_rows == 1 && a.dgate) {
                const float s = a.scale ? a.scale[j] : 1.0f;
                float d = q * s * (a.post ? __builtin_fmaf(hh, a.gamma_h ? a.gamma_h[j] : 1.0f, a.beta_h ? a.beta_h[j] : 0.0f) : hh);
                if (a.sigmoid) d *= gv * (1.0f - gv);
                ((elem_t*)a.dgate)[t * a.ldg + j] = Prec<DT>::from_f32(d);
            }
        }
        if (threadIdx.x == 0) a.averages[t * 2] = c1, a.averages[t * 2 + 1] = c2;
        __syncthreads();
    }
}

// The four column sums of each item where no registers held them: a thread eight columns.
template <int DT>
__global__ __launch_bounds__(256) void residual_norm_sums(ResidualNormArgs a)
{
    typedef typename Prec<DT>::elem_t elem_t;
    const int64_t j = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (j >= a.cols) return;
    const int have = (int)min((int64_t)8, a.cols - j);
    float gamma[8], dg[8], db[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) gamma[k] = a.gamma && k < have ? a.gamma[j + k] : 1.0f, dg[k] = db[k] = 0.0f;
    for (int64_t item = blockIdx.y; item < a.items; item += gridDim.y) {
        int64_t first, last;
        item_rows(a, item, first, last);
        float s1[8], s2[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) s1[k] = s2[k] = 0.0f;
        for (int64_t t = first; t < last; ++t) {
            const float4 st = stats_of(a, t);
            const float c1 = a.averages[t * 2], c2 = a.averages[t * 2 + 1];
            float q[8], x[8], dy[8], h[8], g[8];
            if (a.dr_out) get8<DT>(a.dr_out, t * a.ldr + j, q, have);
            if (a.dy) get8<DT>(a.x, t * a.ldr + j, x, have), get8<DT>(a.dy, t * a.ldy + j, dy, have);
            get8<DT>(a.h, t * a.ldh + j, h, have);
            const bool own_gate = a.gate && a.gate_rows == 1;
            if (own_gate) get8<DT>(a.gate, t * a.ldg + j, g, have);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (!a.dr_out) q[k] = 0.0f;
                if (a.dy) {
                    const float xh = (x[k] - st.z) * st.w;
                    dg[k] = __builtin_fmaf(dy[k], xh, dg[k]), db[k] += dy[k];
                    q[k] += st.w * (dy[k] * gamma[k] - c1 - xh * c2);
                }
                if (own_gate) q[k] *= gate_of(g[k], a.sigmoid);
                s1[k] += q[k], s2[k] = __builtin_fmaf(q[k], a.post ? (h[k] - st.x) * st.y : h[k], s2[k]);
            }
        }
        if (a.sums_h) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < have) a.sums_h[item * 2 * a.cols + j + k] = s1[k], a.sums_h[item * 2 * a.cols + a.cols + j + k] = s2[k];
        }
    }
    if (a.sums) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < have) a.sums[(int64_t)blockIdx.y * 2 * a.cols + j + k] = dg[k], a.sums[(int64_t)blockIdx.y * 2 * a.cols + a.cols + j + k] = db[k];
    }
}

// ---- joins ----------------------------------------------------------------------------------------------------------------

// What the gates' gradient takes: scale, gamma_h and beta_h of a column.
struct Column {
    float s, ga, gb;
    __device__ __forceinline__ Column(const ResidualNormArgs& a, int j)
        : s(a.scale ? a.scale[j] : 1.0f), ga(a.post && a.gamma_h ? a.gamma_h[j] : 1.0f), gb(a.post && a.beta_h ? a.beta_h[j] : 0.0f)
    {
    }
};
// The sums of every `step`-th run from `first` of gate row g, which rows share.
__device__ __forceinline__ void runs_of_gate(const ResidualNormArgs& a, int64_t g, int first, int step, int j, float& s1, float& s2)
{
    s1 = s2 = 0.0f;
#pragma unroll 4
    for (int p = first; p < a.per; p += step) s1 += a.sums_h[(g * a.per + p) * 2 * a.cols + j], s2 += a.sums_h[(g * a.per + p) * 2 * a.cols + a.cols + j];
}
// Its gradient from the sums of all of its runs, which become those of its rows times the gate.
template <int DT>
__device__ __forceinline__ void gate_row(const ResidualNormArgs& a, const Column& c, int64_t g, int j, float& s1, float& s2)
{
    typedef typename Prec<DT>::elem_t elem_t;
    const float gate = gate_of(Prec<DT>::to_f32(((const elem_t*)a.gate)[g * a.ldg + j]), a.sigmoid);
    if (a.dgate) {
        float d = c.s * __builtin_fmaf(c.ga, s2, c.gb * s1);
        if (a.sigmoid) d *= gate * (1.0f - gate);
        ((elem_t*)a.dgate)[g * a.ldg + j] = Prec<DT>::from_f32(d);
    }
    s1 *= gate, s2 *= gate;
}

// Many gate rows: a kernel of their own, which leaves the sums times the gate at the gate's first run.
template <int DT>
__global__ __launch_bounds__(256) void residual_norm_gates(ResidualNormArgs a)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= a.cols) return;
    const Column c(a, j);
    const int64_t gates = a.items / a.per;
    for (int64_t g = blockIdx.y; g < gates; g += gridDim.y) {
        float s1, s2;
        runs_of_gate(a, g, 0, 1, j, s1, s2);
        gate_row<DT>(a, c, g, j, s1, s2);
        a.sums_h[g * a.per * 2 * a.cols + j] = s1, a.sums_h[g * a.per * 2 * a.cols + a.cols + j] = s2;
    }
}

// Sums of `parts` and of `items` (every `per`-th run, or GATES: gate rows), C columns and 1024 / C lanes of rows a workgroup, and from them the gradients
// of the vectors.
template <int DT, bool GATES, int C>
__global__ __launch_bounds__(1024) void residual_norm_join(ResidualNormArgs a, int parts, int64_t items, int per)
{
    constexpr int LANES = 1024 / C;
    __shared__ float red[4][LANES][C];
    const int l = threadIdx.x % C, lane = threadIdx.x / C;
    const int j = blockIdx.x * C + l;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    // lanes that share a gate row's runs, where there are fewer gate rows than lanes (999 x 1000 bf16 with one gate row: 27.4 us with a lane a gate row, 20.9 so)
    const int share = GATES && 2 * items <= LANES ? LANES / (int)items : 1;
    if (j < a.cols) {
        if (a.sums) {
#pragma unroll 4
            for (int p = lane; p < parts; p += LANES) s[0] += a.sums[(int64_t)p * 2 * a.cols + j], s[1] += a.sums[(int64_t)p * 2 * a.cols + a.cols + j];
        }
        if constexpr (GATES) {
            if (share == 1) {
                const Column c(a, j);
                for (int64_t g = lane; g < items; g += LANES) {
                    float s1, s2;
                    runs_of_gate(a, g, 0, 1, j, s1, s2);
                    gate_row<DT>(a, c, g, j, s1, s2);
                    s[2] += s1, s[3] += s2;
                }
            } else if (lane / share < items) {
                runs_of_gate(a, lane / share, lane % share, share, j, s[2], s[3]);
            }
        } else if (a.sums_h) {
#pragma unroll 4
            for (int64_t p = lane; p < items; p += LANES) s[2] += a.sums_h[p * per * 2 * a.cols + j], s[3] += a.sums_h[p * per * 2 * a.cols + a.cols + j];
        }
    }
    if (GATES && share > 1) {
        red[2][lane][l] = s[2], red[3][lane][l] = s[3];
        __syncthreads();
        float s1 = 0.0f, s2 = 0.0f;
        if (lane < items && j < a.cols) {
            for (int p = lane * share; p < (lane + 1) * share; ++p) s1 += red[2][p][l], s2 += red[3][p][l];
            gate_row<DT>(a, Column(a, j), lane, j, s1, s2);
        }
        s[2] = s1, s[3] = s2;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) red[i][lane][l] = s[i];
    __syncthreads();
    if (lane >= 4) return;
    float sum = 0.0f;  // lane i: sum i
#pragma unroll 16
    for (int p = 0; p < LANES; ++p) sum += red[lane][p][l];
    if (j >= a.cols) return;
    const Column c(a, j);
    if (lane == 0 && a.dgamma) a.dgamma[j] = sum;
    if (lane == 1 && a.dbeta) a.dbeta[j] = sum;
    if (lane == 2 && a.dbeta_h) a.dbeta_h[j] = c.s * sum;
    if (lane == 3 && a.dgamma_h) a.dgamma_h[j] = c.s * sum;
    if (lane == 3 && a.dscale) {
        float s1 = 0.0f;  // (the same sum as lane 2's)
#pragma unroll 16
        for (int p = 0; p < LANES; ++p) s1 += red[2][p][l];
        a.dscale[j] = __builtin_fmaf(c.ga, sum, c.gb * s1);
    }
}

// 64 columns a workgroup where that leaves some for every CU, else 16.
template <int DT, bool GATES>
void join(const ResidualNormArgs& a, int parts, int64_t items, int per, hipStream_t s)
{
    if (a.cols >= 16 * kCUs) hipLaunchKernelGGL((residual_norm_join<DT, GATES, 64>), dim3((unsigned)((a.cols + 63) / 64)), dim3(1024), 0, s, a, parts, items, per);
    else hipLaunchKernelGGL((residual_norm_join<DT, GATES, 16>), dim3((unsigned)((a.cols + 15) / 16)), dim3(1024), 0, s, a, parts, items, per);
}

// ---- forms ----------------------------------------------------------------------------------------------------------------

ResidualNormForm fwd_form(int cols, int dtype)
{
    const int vec = dtype == CONV_F32 ? 4 : 8;
    ResidualNormForm f = {};
    if (vec == 4 && cols <= 32) f.lanes = 8, f.most = 4, f.waves = 4;
    for (int lanes : {8, 16, 64})
        for (int most : {8, 16})
            if (cols <= lanes * most && !f.lanes) f.lanes = lanes, f.most = most, f.waves = 4;
    if (f.lanes) return f;
    const int pieces = (cols + vec - 1) / vec;
    for (int most : {8, 16}) {
        const int waves = (pieces + 64 * (most / vec) - 1) / (64 * (most / vec));
        if (waves <= (most == 8 ? 8 : 16)) {
            f.lanes = 64 * waves, f.most = most, f.waves = waves;
            return f;
        }
    }
    return f;  // none
}

// Backward: lanes a row and elements a lane; workgroups, and the runs of rows that they take.
ResidualNormForm bwd_form(int64_t rows, int cols, int64_t gate_rows, int dtype)
{
    ResidualNormForm f = {};
    if (dtype == CONV_F32 && cols <= 32) f.lanes = 8, f.most = 4;
    for (int lanes = 8; lanes <= 1024 && !f.lanes; lanes *= 2)
        if (cols <= lanes * 8) f.lanes = lanes, f.most = 8;
    if (!f.lanes && cols <= 16384) f.lanes = 1024, f.most = 16;
    f.sums = f.most == 16 || !f.lanes;  // the column sums by a kernel of their own
    const int here = f.sums ? 1 : (f.lanes <= 256 ? 256 : f.lanes) / f.lanes;  // rows at once
    const int64_t most = f.sums ? 128 : f.lanes >= 512 ? kCUs : f.lanes <= 16 ? 4 * kCUs : 2 * kCUs;
    f.stretch = std::max<int64_t>(gate_rows > 1 ? std::min(gate_rows, rows) : rows, 1);  // (a gate may stand for more rows than there are)
    const int64_t stretches = (rows + f.stretch - 1) / f.stretch;
    // as many runs as workgroups, of whole rounds; at least eight rows each, lest their sums cost more than they
    const int64_t want = stretches ? std::max<int64_t>(1, most / stretches) : 1;
    const int64_t least = std::max(here, 8);
    f.each = std::max((f.stretch + want - 1) / want, least);
    f.each = (f.each + here - 1) / here * here;
    f.per = (int)((f.stretch + f.each - 1) / f.each);
    f.items = stretches * f.per;
    f.groups = (int)std::min<int64_t>(std::max<int64_t>(f.items, 1), most);
    return f;
}

struct Space {
    float *sums, *sums_h, *averages;
    size_t bytes;
};
Space space_of(const ResidualNormForm& f, int64_t rows, int cols, void* ws)
{
    Space s = {};
    char* at = (char*)ws;
    auto take = [&](size_t n) {
        float* p = at ? (float*)(at + s.bytes) : nullptr;
        s.bytes += (n + 255) & ~(size_t)255;
        return p;
    };
    s.sums = take((size_t)f.groups * 2 * cols * 4);
    s.sums_h = take((size_t)f.items * 2 * cols * 4);
    if (f.sums) s.averages = take((size_t)rows * 2 * 4);
    return s;
}

template <int DT>
hipError_t bwd(ResidualNormArgs a, const ResidualNormForm& f, hipStream_t s)
{
    if (a.rows > 0) {
        if (f.lanes) {
            ResidualNormArgs rows = a;
            ResidualNormForm form = f;
            // Without column sums a workgroup's rows need be neither of one gate nor many: as many workgroups as CUs (the runs of the sums' kernel, 128 at most,
            // left half of them idle)
            if (f.sums) {
                rows.stretch = a.rows, rows.each = (a.rows + kCUs - 1) / kCUs;
                rows.items = (a.rows + rows.each - 1) / rows.each;
                rows.per = form.groups = (int)rows.items;
            }
            const hipError_t e = DT == CONV_F32   ? residual_norm_bwd_f32(rows, form, s)
                                 : DT == CONV_F16 ? residual_norm_bwd_f16(rows, form, s)
                                                  : residual_norm_bwd_bf16(rows, form, s);
            if (e != hipSuccess) return e;
        } else {
            hipLaunchKernelGGL((residual_norm_bwd_any<DT>), dim3((unsigned)std::min<int64_t>(a.rows, 1 << 20)), dim3(1024), 0, s, a);
        }
        if (f.sums && (a.sums || a.sums_h)) hipLaunchKernelGGL((residual_norm_sums<DT>), dim3((unsigned)((a.cols + 2047) / 2048), (unsigned)f.groups), dim3(256), 0, s, a);
    }
    if (!a.sums && !a.sums_h) return hipGetLastError();
    const bool shared = a.rows && a.gate && a.gate_rows > 1 && a.sums_h;
    const int parts = a.rows ? f.groups : 0;
    // few gate rows in the join itself; many by a kernel that has more than a workgroup for 16 columns
    if (shared && f.items / f.per <= 256) {
        join<DT, true>(a, parts, f.items / f.per, f.per, s);
    } else {
        if (shared)
            hipLaunchKernelGGL((residual_norm_gates<DT>), dim3((unsigned)((a.cols + 255) / 256), (unsigned)std::min<int64_t>(f.items / f.per, 4096)), dim3(256), 0, s, a);
        join<DT, false>(a, parts, a.rows ? (shared ? f.items / f.per : f.items) : 0, shared ? f.per : 1, s);
    }
    return hipGetLastError();
}

}  // namespace

size_t residual_norm_bwd_workspace(int64_t rows, int cols, int64_t gate_rows, int dtype)
{
    return space_of(bwd_form(rows, cols, gate_rows, dtype), rows, cols, nullptr).bytes;
}

hipError_t launch_residual_norm_fwd(const ResidualNormArgs& a, int dtype, hipStream_t s)
{
    const ResidualNormForm f = fwd_form(a.cols, dtype);
    if (f.lanes) return dtype == CONV_F32 ? residual_norm_fwd_f32(a, f, s) : dtype == CONV_F16 ? residual_norm_fwd_f16(a, f, s) : residual_norm_fwd_bf16(a, f, s);
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, 1 << 20));
    if (dtype == CONV_F32) hipLaunchKernelGGL((residual_norm_fwd_any<CONV_F32>), grid, dim3(1024), 0, s, a);
    else if (dtype == CONV_F16) hipLaunchKernelGGL((residual_norm_fwd_any<CONV_F16>), grid, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((residual_norm_fwd_any<CONV_BF16>), grid, dim3(1024), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_residual_norm_bwd(ResidualNormArgs& a, int dtype, hipStream_t s)
{
    const ResidualNormForm f = bwd_form(a.rows, a.cols, a.gate ? a.gate_rows : 0, dtype);
    const Space space = space_of(f, a.rows, a.cols, a.ws);
    a.stretch = f.stretch, a.each = f.each, a.items = f.items, a.per = f.per;
    a.sums = a.dgamma || a.dbeta ? space.sums : nullptr;
    a.sums_h = a.dgamma_h || a.dbeta_h || a.dscale || (a.dgate && a.gate_rows > 1) ? space.sums_h : nullptr;
    a.averages = space.averages;
    return dtype == CONV_F32 ? bwd<CONV_F32>(a, f, s) : dtype == CONV_F16 ? bwd<CONV_F16>(a, f, s) : bwd<CONV_BF16>(a, f, s);
}

}  // namespace convfwd
