// Products of fp32 rows: the tiles of linear layers and their gradients.
#include "product_f32_kernel.h"

namespace convfwd {

namespace {

template <typename T, bool A_ACROSS, bool B_ACROSS, bool PARTIAL>
hipError_t launch_tiles(SplitArgs g, const LinearOut& e, int splits, hipStream_t s)
{
    const hipError_t err = ensure_dynamic_lds((const void*)product_f32_kernel<T, A_ACROSS, B_ACROSS, PARTIAL>, T::LDS);
    if (err != hipSuccess) return err;
    g.tiles_n = (int)((g.N + T::BN - 1) / T::BN);
    // a launch holds less than 2^32 threads: the rows go in portions of so many tiles
    const int64_t all = g.M, bands = std::max<int64_t>(1, (1 << 21) / ((int64_t)g.tiles_n * splits));
    for (int64_t skip = 0; skip < all; skip += bands * T::BT) {
        SplitArgs p = g;
        p.M = std::min(bands * T::BT, all - skip), p.m_first = skip;
        p.a += A_ACROSS ? skip : skip * g.lda;
        p.tiles_m = (int)((p.M + T::BT - 1) / T::BT);
        hipLaunchKernelGGL((product_f32_kernel<T, A_ACROSS, B_ACROSS, PARTIAL>), dim3((unsigned)p.tiles_m * (unsigned)p.tiles_n * (unsigned)splits), dim3(T::NT), T::LDS, s,
                           p, e);
    }
    return hipGetLastError();
}

template <typename T, bool PARTIAL>
hipError_t launch_layout(const SplitArgs& g, const LinearOut& e, ProductLayout layout, int splits, hipStream_t s)
{
    switch (layout) {
        case LAYOUT_NT: return launch_tiles<T, false, false, PARTIAL>(g, e, splits, s);
        case LAYOUT_NN: return launch_tiles<T, false, true, PARTIAL>(g, e, splits, s);
        default: return launch_tiles<T, true, true, PARTIAL>(g, e, splits, s);
    }
}

}  // namespace

hipError_t launch_product_f32(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s)
{
    SplitArgs p = {};
    p.a = (const float*)g.a, p.b = (const float*)g.b, p.lda = g.lda, p.ldb = g.ldb, p.M = g.M, p.N = g.N, p.K = g.K, p.partial = g.partial;
    p.each = (int64_t)((g.ksteps + splits - 1) / splits) * 64, p.splits = splits;
    typedef SplitTile<2, 2, 2, 2> Tile64;
    typedef SplitTile<2, 4, 4, 2> Tile128;
    typedef SplitTile<4, 2, 4, 4> Tile256;
    switch (form) {
        case P64: return splits > 1 ? launch_layout<Tile64, true>(p, e, layout, splits, s) : launch_layout<Tile64, false>(p, e, layout, splits, s);
        case P128: return splits > 1 ? launch_layout<Tile128, true>(p, e, layout, splits, s) : launch_layout<Tile128, false>(p, e, layout, splits, s);
        default: return splits > 1 ? launch_layout<Tile256, true>(p, e, layout, splits, s) : launch_layout<Tile256, false>(p, e, layout, splits, s);
    }
}

}  // namespace convfwd
