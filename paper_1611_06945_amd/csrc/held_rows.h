// Rows held in registers by the lanes that share them, for the operators that normalise rows.
#pragma once

#include "rows_common.h"

namespace convfwd {

// The pieces of a row that a lane holds: lane l of G has pieces l, l + G, ...
template <int DT, int G, int NV>
struct Held {
    typedef typename Prec<DT>::elem_t elem_t;
    typedef Piece<DT> P;
    static constexpr int VEC = P::VEC;
    static __device__ __forceinline__ int lanes() { return G ? G : (int)blockDim.x; }

    // Stored values, one load for every piece and no branch around it: a piece that would pass the row's end is read at the end, and
    // clear() puts it right.  (With a branch for the pieces at the end, which loaded element by element, a wave waited there for all
    // its loads: backward, 65536 x 768 bf16 90 us against 58.)
    static __device__ __forceinline__ void load(uint4 (&raw)[NV], const elem_t* x, int cols, int l)
    {
        if constexpr (G == 8 && NV == 1) {
            if (cols < VEC) {
                elem_t e[VEC];
#pragma unroll
                for (int k = 0; k < VEC; ++k) e[k] = k < cols ? x[k] : (elem_t)0;
                __builtin_memcpy(&raw[0], e, 16);
                return;
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i] = P::raw(x + min((i * lanes() + l) * VEC, cols - VEC));
    }
    // zeros past the end of the row
    static __device__ __forceinline__ void clear(uint4 (&raw)[NV], int cols, int l)
    {
        const int past = cols < VEC ? 0 : -cols & (VEC - 1);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int left = cols - (i * lanes() + l) * VEC;
            uint4 w = raw[i];
            if (past) {
                const uint4 v = P::shifted(w, past);
                w.x = left < VEC ? v.x : w.x, w.y = left < VEC ? v.y : w.y, w.z = left < VEC ? v.z : w.z, w.w = left < VEC ? v.w : w.w;
            }
            w.x = left > 0 ? w.x : 0, w.y = left > 0 ? w.y : 0, w.z = left > 0 ? w.z : 0, w.w = left > 0 ? w.w : 0;
            raw[i] = w;
        }
    }
    static __device__ __forceinline__ void store(elem_t* y, const float (&v)[VEC], int cols, int i, int l)
    {
        const int j = (i * lanes() + l) * VEC;
        const uint4 u = P::narrow(v);
        if (j + VEC <= cols) {
            P::put(y + j, u);
        } else if (j < cols) {
            elem_t e[VEC];
            __builtin_memcpy(e, &u, 16);
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (j + k < cols) y[j + k] = e[k];
        }
    }
    // a vector over the columns, `none` where the pointer is null or the row has ended
    static __device__ __forceinline__ void columns(float (&v)[NV][VEC], const float* p, float none, int cols, int l)
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = (i * lanes() + l) * VEC;
            if (p && j + VEC <= cols) {
                __builtin_memcpy(v[i], p + j, 4 * VEC);
            } else {
#pragma unroll
                for (int k = 0; k < VEC; ++k) v[i][k] = p && j + k < cols ? p[j + k] : none;
            }
        }
    }
};

// Combines a value over the lanes of a row; `lds` holds a float for each wave of the workgroup and call within a row.  (Sums or largest
// magnitudes: zero is neutral.)
template <int G, typename Op>
__device__ __forceinline__ float row_reduce(float x, float* lds)
{
    if constexpr (G > 0) {
        return lanes_reduce<G, Op>(x);
    } else {
        // waves as many as the workgroup has, up to 16: each reads what all left behind
        x = lanes_reduce<64, Op>(x);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        const int w = threadIdx.x & 15;
        return lanes_reduce<16, Op>(w < (int)(blockDim.x >> 6) ? lds[w] : 0.0f);
    }
}

}  // namespace convfwd
