// Newton-Schulz steps that bring the singular values of a matrix towards one, as an update's direction is made orthogonal.
//
//   X = x / (|x| + eps);  `steps` times:  A = X X^T,  B = b A + c A A,  X <- a X + B X      (A = X^T X, X <- a X + X B where X is tall)
//
// A and B have the side of the shorter dimension n and are symmetric: only the tiles on and above the diagonal are multiplied, each written to both its
// places, so a step takes n n (3 m + n) operations for the longer dimension m.  All products are those of product_kernel.h, on fp16 operands scaled by
// 2^12 (X, A and B are small whole numbers at most and their elements of the size 1 / sqrt(n): scaled they keep all their bits).
//   * X itself is kept in more bits than it is multiplied in: weak directions grow by a in every step, and so would the roundings of an X kept in 16
//     bits (a matrix of rank n / 8 in bf16: 3 % off, against 0.08 %).  The errors of A, B and the X that B multiplies do not grow like that.
//   * The products take two planes of each operand, high and low, and three of their four products: 22 bits.  One plane, 11 bits, is three times as fast, but leaves a
//     bf16 result off by up to 2.1 times its own rounding, most where all singular values are alike (orthonormal 141 x 141 in five steps; normal ones 1.5; some strong directions
//     above weak ones 1.1 to 1.3), and the steps' slopes let errors of early steps grow in late ones.  Even the first step alone in one plane counts where one
//     direction is nearly all of x (700 x 700 of rank one 1.15).
//   * Bound by the products where there are tiles for all CUs (4096 x 4096 bf16, five steps, traced: 241, 245 and 345 us for the three products of a step, 29 before them, 4184 in
//     all; 4120 to 4220 without the trace, 0.99 PFLOP/s), by 17 launches one after the other where there are not (24 of 192 x 768 fp32: 11, 7 and 23 us a step, 213 in all).
//   * X beside its products: fp32 for fp32; for 16-bit types the high and the low plane together, 22 bits, which is less to read and write.
#include <algorithm>
#include <cmath>

#include "linear_common.h"

namespace convfwd {

namespace {

constexpr float kPlane = 0x1p12f, kUnplane = 0x1p-12f;

// A matrix of the workspace in fp16 planes: planes [planes][rows][ld] for each matrix of the batch.
struct Planes {
    uint16_t* p;
    int64_t ld, plane, batch;
};

// eight values, scaled, as high and low planes
__device__ __forceinline__ void split2(const float (&v)[8], float (&hi)[8], float (&lo)[8])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint16_t h = Prec<CONV_F16>::from_f32(v[k]);
        hi[k] = Prec<CONV_F16>::to_f32(h), lo[k] = v[k] - hi[k];
    }
}
__device__ __forceinline__ void put_scaled(const Planes& to, int64_t row, int64_t col, const float (&v)[8], int have)
{
    uint16_t* const p = to.p + blockIdx.y * to.batch;
    float hi[8], lo[8];
    split2(v, hi, lo);
    put8<CONV_F16>(p, row * to.ld + col, hi, have);
    put8<CONV_F16>(p + to.plane, row * to.ld + col, lo, have);
}
// ... and to the place mirrored at the diagonal: neighbouring lanes have neighbouring rows, which lie next to each other there
__device__ __forceinline__ void put_mirrored(const Planes& to, int64_t row, int64_t col, const float (&v)[8], int have)
{
    uint16_t* const p = to.p + blockIdx.y * to.batch + col * to.ld + row;
    float hi[8], lo[8];
    split2(v, hi, lo);
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < have) {
            p[k * to.ld] = Prec<CONV_F16>::from_f32(hi[k]);
            p[to.plane + k * to.ld] = Prec<CONV_F16>::from_f32(lo[k]);
        }
}
__device__ __forceinline__ void get_scaled(const Planes& from, int64_t row, int64_t col, float (&v)[8], int have)
{
    const uint16_t* const p = from.p + blockIdx.y * from.batch;
    float lo[8];
    get8<CONV_F16>(p, row * from.ld + col, v, have);
    get8<CONV_F16>(p + from.plane, row * from.ld + col, lo, have);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += lo[k];
}

struct GramEpi {
    struct Args {
        Planes a;
        int side;  // of the tiles
    };
    static constexpr bool SYMMETRIC = true;
    static __device__ __forceinline__ void prepare(const Args&, float*, int64_t, int, int, int) {}
    static __device__ __forceinline__ void finish(const ProductArgs&, const Args& e, float (&v)[8], int64_t m, int64_t n, int have, const float*)
    {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= kUnplane;
        put_scaled(e.a, m, n, v, have);
        if ((uint32_t)m / (uint32_t)e.side != (uint32_t)n / (uint32_t)e.side) put_mirrored(e.a, m, n, v, have);
    }
};

struct SquareEpi {
    struct Args {
        Planes a, b;
        float coef_b, coef_c;
        int side;  // of the tiles
    };
    static constexpr bool SYMMETRIC = true;
    static __device__ __forceinline__ void prepare(const Args&, float*, int64_t, int, int, int) {}
    static __device__ __forceinline__ void finish(const ProductArgs&, const Args& e, float (&v)[8], int64_t m, int64_t n, int have, const float*)
    {
        float a[8];
        get_scaled(e.a, m, n, a, have);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __builtin_fmaf(e.coef_b, a[k], e.coef_c * kUnplane * v[k]);
        put_scaled(e.b, m, n, v, have);
        if ((uint32_t)m / (uint32_t)e.side != (uint32_t)n / (uint32_t)e.side) put_mirrored(e.b, m, n, v, have);
    }
};

struct UpdateEpi {
    struct Args {
        float* x;        // in fp32, [rows][ld of the planes]; null: the planes hold it
        int64_t batch_x;
        Planes from, to;
        float coef_a;
        void* out;       // the last step's result, instead of the planes
        int64_t ldo, batch_o;
        int dtype;
    };
    static constexpr bool SYMMETRIC = false;
    static __device__ __forceinline__ void prepare(const Args&, float*, int64_t, int, int, int) {}
    static __device__ __forceinline__ void finish(const ProductArgs&, const Args& e, float (&v)[8], int64_t m, int64_t n, int have, const float*)
    {
        float* const x = e.x + blockIdx.y * e.batch_x;
        float old[8], scale = e.coef_a;
        if (e.x) get8<CONV_F32>(x, m * e.to.ld + n, old, have);
        else get_scaled(e.from, m, n, old, have), scale *= kUnplane;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __builtin_fmaf(scale, old[k], kUnplane * kUnplane * v[k]);
        if (!e.out) {
            if (e.x) put8<CONV_F32>(x, m * e.to.ld + n, v, have);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= kPlane;
            put_scaled(e.to, m, n, v, have);
        } else {
            const int64_t at = blockIdx.y * e.batch_o + m * e.ldo + n;
            if (e.dtype == CONV_F32) put8<CONV_F32>(e.out, at, v, have);
            else if (e.dtype == CONV_F16) put8<CONV_F16>(e.out, at, v, have);
            else put8<CONV_BF16>(e.out, at, v, have);
        }
    }
};

struct StartArgs {
    const void* x;
    int64_t ldx, stride_x;
    int64_t rows, cols;
    double* sums;                  // [batch][parts]
    int parts;
    float* x32;
    int64_t batch_x;
    Planes to;
    double eps;
};

// The sum of the squares in doubles, in which no fp32 value's square overflows or vanishes.
template <int DT>
__global__ __launch_bounds__(256) void orthogonal_norm(StartArgs g)
{
    typedef typename Prec<DT>::elem_t elem_t;
    __shared__ double red[256];
    const elem_t* x = (const elem_t*)g.x + blockIdx.y * g.stride_x;
    const int64_t each = (g.cols + 7) / 8, all = g.rows * each, step = (int64_t)gridDim.x * 256;
    double sum = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const int64_t t = all <= UINT32_MAX ? (uint32_t)i / (uint32_t)each : i / each, j = (i - t * each) * 8;
        float v[8];
        get8<DT>(x, t * g.ldx + j, v, (int)min(g.cols - j, (int64_t)8));
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += (double)v[k] * v[k];
    }
    red[threadIdx.x] = sum;
    __syncthreads();
    for (int half = 128; half >= 1; half /= 2) {
        if ((int)threadIdx.x < half) red[threadIdx.x] += red[threadIdx.x + half];
        __syncthreads();
    }
    if (threadIdx.x == 0) g.sums[blockIdx.y * g.parts + blockIdx.x] = red[0];
}

// X in planes, and in fp32 where it is kept so.
template <int DT>
__global__ __launch_bounds__(256) void orthogonal_start(StartArgs g)
{
    typedef typename Prec<DT>::elem_t elem_t;
    __shared__ double red[256];
    double sum = 0.0;
    for (int p = threadIdx.x; p < g.parts; p += 256) sum += g.sums[blockIdx.y * g.parts + p];
    red[threadIdx.x] = sum;
    __syncthreads();
    for (int half = 128; half >= 1; half /= 2) {
        if ((int)threadIdx.x < half) red[threadIdx.x] += red[threadIdx.x + half];
        __syncthreads();
    }
    const double inv = 1.0 / (sqrt(red[0]) + g.eps);
    const elem_t* x = (const elem_t*)g.x + blockIdx.y * g.stride_x;
    float* x32 = g.x32 + blockIdx.y * g.batch_x;
    const int64_t ld = g.to.ld, each = ld / 8, all = g.rows * each, step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t i = first; i < all; i += step) {
        const int64_t t = all <= UINT32_MAX ? (uint32_t)i / (uint32_t)each : i / each, j = (i - t * each) * 8;
        const int have = (int)min(g.cols - j, (int64_t)8);
        float v[8];
        get8<DT>(x, t * g.ldx + j, v, have);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (float)(v[k] * inv);
        if (g.x32) put8<CONV_F32>(x32, t * ld + j, v, have);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= kPlane;
        put_scaled(g.to, t, j, v, have);
    }
}

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

int parts_of(int64_t rows, int64_t cols) { return (int)std::max<int64_t>(1, std::min<int64_t>(1024, rows * cols / 8192)); }

struct Space {
    Planes x[2], a, b;
    float* x32;
    int64_t batch_x;
    double* sums;
    size_t bytes;
};
Space space_of(const OrthogonalArgs& g, int dtype, void* ws)
{
    Space s = {};
    char* at = (char*)ws;
    auto take = [&](size_t n) {
        char* p = at ? at + s.bytes : nullptr;
        s.bytes += (n + 255) & ~(size_t)255;
        return (void*)p;
    };
    auto matrix = [&](int64_t rows, int64_t cols) {
        Planes p = {};
        p.ld = round_up(cols, 8), p.plane = rows * p.ld, p.batch = p.plane * 2;
        p.p = (uint16_t*)take((size_t)g.batch * p.batch * 2);
        return p;
    };
    const int64_t side = std::min(g.rows, g.cols);
    s.x[0] = matrix(g.rows, g.cols), s.x[1] = matrix(g.rows, g.cols);
    s.a = matrix(side, side), s.b = matrix(side, side);
    s.batch_x = g.rows * s.x[0].ld;
    if (dtype == CONV_F32) s.x32 = (float*)take((size_t)g.batch * s.batch_x * 4);
    s.sums = (double*)take((size_t)g.batch * parts_of(g.rows, g.cols) * 8);
    return s;
}

// Tiles of two planes.
typedef ProductTile<4, 2, 1, 2, 2, 2> Tile64Two;      // two workgroups a CU
typedef ProductTile<4, 2, 1, 2, 4, 2> Tile64TwoDeep;  // one: three steps on their way (4 of 2048 x 512 fp16: 307 -> 268 us)
typedef ProductTile<2, 4, 4, 2, 2, 2> Tile128Two;
struct TileCost {
    int side;
    double once, own, step;
    bool alone;  // for a workgroup a CU at most, and more steps than it has stages (12 of 192 x 192: 114 us, with it 116)
};
constexpr TileCost kTiles[] = {{64, 4.1, 1.0, 0.5, false}, {128, 3.1, 3.0, 1.3, false}, {64, 4.1, 1.0, 0.4, true}};
enum TileId { T64, T128, T64_DEEP };

// The tile with the least expected time, in us (see the linear layers' plan).
TileId tile_of(int64_t M, int64_t N, int64_t K, int64_t batch, bool symmetric)
{
    int best = 0;
    double least = 1e30;
    for (int f = 0; f < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++f) {
        const TileCost& c = kTiles[f];
        const double tm = (double)((M + c.side - 1) / c.side), tn = (double)((N + c.side - 1) / c.side);
        const double tiles = (symmetric ? tm * (tm + 1) / 2 : tm * tn) * batch, steps = (double)((K + 63) / 64);
        const double us = c.once + std::ceil(tiles / 256) * (c.own + steps * c.step);
        if (c.alone && (tiles > 256 || steps <= 4)) continue;
        if (us < least) least = us, best = f;
    }
    return (TileId)best;
}
int64_t tiles_of(TileId f, int64_t M, int64_t N)
{
    const int side = kTiles[f].side;
    return ((M + side - 1) / side) * ((N + side - 1) / side);
}

template <bool A_ACROSS, bool B_ACROSS, typename Epi>
hipError_t multiply(const ProductArgs& g, const typename Epi::Args& e, TileId tile, int batch, hipStream_t s)
{
    switch (tile) {
        case T64: return launch_product_tiles<CONV_F16, Tile64Two, A_ACROSS, B_ACROSS, true, Epi>(g, e, batch, 1, s);
        case T128: return launch_product_tiles<CONV_F16, Tile128Two, A_ACROSS, B_ACROSS, true, Epi>(g, e, batch, 1, s);
        default: return launch_product_tiles<CONV_F16, Tile64TwoDeep, A_ACROSS, B_ACROSS, true, Epi>(g, e, batch, 1, s);
    }
}

ProductArgs product_of(const Planes& a, const Planes& b, int64_t M, int64_t N, int64_t K)
{
    ProductArgs p = {};
    p.a = a.p, p.b = b.p, p.lda = a.ld, p.ldb = b.ld, p.plane_a = a.plane, p.plane_b = b.plane, p.batch_a = a.batch, p.batch_b = b.batch;
    p.M = M, p.N = N, p.K = K, p.ksteps = (int)((K + 63) / 64);
    return p;
}

template <int DT>
hipError_t start(const StartArgs& g, int64_t batch, hipStream_t s)
{
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(2048, g.rows * g.to.ld / 2048));
    hipLaunchKernelGGL((orthogonal_norm<DT>), dim3((unsigned)g.parts, (unsigned)batch), dim3(256), 0, s, g);
    hipLaunchKernelGGL((orthogonal_start<DT>), dim3((unsigned)blocks, (unsigned)batch), dim3(256), 0, s, g);
    return hipGetLastError();
}

}  // namespace

size_t orthogonal_workspace(const OrthogonalArgs& g, int dtype) { return g.batch == 0 ? 0 : space_of(g, dtype, nullptr).bytes; }

hipError_t launch_orthogonalize(const OrthogonalArgs& all, int dtype, hipStream_t s)
{
    // gridDim.y is at most 65535, and a launch holds less than 2^32 threads: the batch goes in portions, tiles chosen for the largest
    const int es = dtype_size(dtype);
    const int64_t side = std::min(all.rows, all.cols), longer = std::max(all.rows, all.cols), most = std::min<int64_t>(all.batch, 32768);
    const TileId gram = tile_of(side, side, longer, most, true), square = tile_of(side, side, side, most, true);
    const TileId update = tile_of(all.rows, all.cols, side, most, false);
    const int64_t tiles = std::max({tiles_of(gram, side, side), tiles_of(square, side, side), tiles_of(update, all.rows, all.cols)});
    const int64_t portion = std::max<int64_t>(1, std::min(most, ((int64_t)1 << 21) / tiles));
    for (int64_t skip = 0; skip < all.batch; skip += portion) {
        OrthogonalArgs g = all;
        g.batch = std::min(portion, all.batch - skip);
        g.x = (const char*)all.x + skip * all.stride_x * es, g.out = (char*)all.out + skip * all.stride_o * es;
        const Space w = space_of(g, dtype, all.ws);
        const bool tall = g.rows > g.cols;
        StartArgs st = {};
        st.x = g.x, st.ldx = g.ldx, st.stride_x = g.stride_x, st.rows = g.rows, st.cols = g.cols, st.sums = w.sums;
        st.parts = parts_of(g.rows, g.cols), st.x32 = w.x32, st.batch_x = w.batch_x, st.to = w.x[0], st.eps = g.eps;
        hipError_t e = dtype == CONV_F32 ? start<CONV_F32>(st, g.batch, s) : dtype == CONV_F16 ? start<CONV_F16>(st, g.batch, s) : start<CONV_BF16>(st, g.batch, s);
        if (e != hipSuccess) return e;
        const int batch = (int)g.batch;
        for (int step = 0; step < g.steps; ++step) {
            const Planes &x = w.x[step & 1], &to = w.x[(step + 1) & 1];
            const GramEpi::Args ge = {w.a, kTiles[gram].side};
            const ProductArgs gp = product_of(x, x, side, side, longer);
            e = tall ? multiply<true, true, GramEpi>(gp, ge, gram, batch, s) : multiply<false, false, GramEpi>(gp, ge, gram, batch, s);
            if (e != hipSuccess) return e;
            const SquareEpi::Args se = {w.a, w.b, g.b, g.c, kTiles[square].side};
            e = multiply<false, false, SquareEpi>(product_of(w.a, w.a, side, side, side), se, square, batch, s);
            if (e != hipSuccess) return e;
            const UpdateEpi::Args ue = {w.x32, w.batch_x, x, to, g.a, step + 1 == g.steps ? g.out : nullptr, g.ldo, g.stride_o, dtype};
            e = tall ? multiply<false, false, UpdateEpi>(product_of(x, w.b, g.rows, g.cols, side), ue, update, batch, s)
                     : multiply<false, true, UpdateEpi>(product_of(w.b, x, g.rows, g.cols, side), ue, update, batch, s);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace convfwd
