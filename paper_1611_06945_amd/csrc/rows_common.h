// Device helpers of the operators on rows: 16-byte pieces of rows that start at any element, reductions over a wave.
#pragma once

#include "igemm_kernel.h"

namespace convfwd {

// 16 bytes of a row: VEC elements of the storage type, as fp32 in registers.  Rows start wherever their stride puts them, so the
// address is only known to be a multiple of the element; global memory takes 16-byte accesses at any such address.
template <int DT>
struct Piece {
    typedef typename Prec<DT>::elem_t elem_t;
    static constexpr int VEC = 16 / (int)sizeof(elem_t);
    static __device__ __forceinline__ uint4 raw(const elem_t* p)
    {
        uint4 v;
        __builtin_memcpy(&v, p, 16);
        return v;
    }
    static __device__ __forceinline__ void widen(const uint4& v, float (&x)[VEC])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if constexpr (DT == CONV_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(float, w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = Prec<DT>::to_f32((elem_t)(w[i] & 0xFFFFu));
                x[2 * i + 1] = Prec<DT>::to_f32((elem_t)(w[i] >> 16));
            }
        }
    }
    static __device__ __forceinline__ uint4 narrow(const float (&x)[VEC])
    {
        if constexpr (DT == CONV_F32)
            return make_uint4(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]), __builtin_bit_cast(uint32_t, x[2]),
                              __builtin_bit_cast(uint32_t, x[3]));
        else
            return make_uint4(Prec<DT>::pack2_from_f32(x[0], x[1]), Prec<DT>::pack2_from_f32(x[2], x[3]),
                              Prec<DT>::pack2_from_f32(x[4], x[5]), Prec<DT>::pack2_from_f32(x[6], x[7]));
    }
    static __device__ __forceinline__ void put(elem_t* p, const uint4& v) { __builtin_memcpy(p, &v, 16); }
    // A row's last piece, where it is short, is read so that it ends with the row, without a branch.  Its first `past` elements are then
    // another piece's: the others come to the front, zeros follow.  (`past` is the same in all lanes: 0 .. VEC - 1.)
    static __device__ __forceinline__ uint4 shifted(const uint4& u, int past)
    {
        const int words = past * (int)sizeof(elem_t) / 4;
        uint32_t v[5] = {u.x, u.y, u.z, u.w, 0};
        if (words & 2) v[0] = v[2], v[1] = v[3], v[2] = v[3] = 0;
        if (words & 1) v[0] = v[1], v[1] = v[2], v[2] = v[3], v[3] = 0;
        if (VEC == 8 && (past & 1)) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = __builtin_amdgcn_alignbit(v[k + 1], v[k], 16);
        }
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
};

// W neighbouring elements, whole pieces (n of them exist), to or from a row that starts at any element.
template <int DT, int W>
__device__ __forceinline__ void put_pieces(void* row, int64_t at, const float (&v)[W], int n)
{
    typedef Piece<DT> P;
    typename P::elem_t* p = (typename P::elem_t*)row + at;
    constexpr int VEC = P::VEC;
#pragma unroll
    for (int c = 0; c < W / VEC; ++c) {
        float part[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) part[k] = v[c * VEC + k];
        const uint4 u = P::narrow(part);
        if (n >= (c + 1) * VEC) {
            P::put(p + c * VEC, u);
        } else {
            typename P::elem_t e[VEC];
            __builtin_memcpy(e, &u, 16);
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                if (c * VEC + k < n) p[c * VEC + k] = e[k];
        }
    }
}
template <int DT, int W>
__device__ __forceinline__ void get_pieces(const void* row, int64_t at, float (&v)[W], int n)
{
    typedef Piece<DT> P;
    const typename P::elem_t* p = (const typename P::elem_t*)row + at;
    constexpr int VEC = P::VEC;
#pragma unroll
    for (int c = 0; c < W / VEC; ++c) {
        if (n >= (c + 1) * VEC) {
            float part[VEC];
            P::widen(P::raw(p + c * VEC), part);
#pragma unroll
            for (int k = 0; k < VEC; ++k) v[c * VEC + k] = part[k];
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k) v[c * VEC + k] = c * VEC + k < n ? Prec<DT>::to_f32(p[c * VEC + k]) : 0.0f;
        }
    }
}

// ... eight of them
template <int DT>
__device__ __forceinline__ void put8(void* row, int64_t at, const float (&v)[8], int n) { put_pieces<DT, 8>(row, at, v, n); }
template <int DT>
__device__ __forceinline__ void get8(const void* row, int64_t at, float (&v)[8], int n) { get_pieces<DT, 8>(row, at, v, n); }

struct OpSum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct OpMax {  // of values that are not NaN
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};

// x combined over groups of G neighbouring lanes (G a power of two up to 64); every lane gets the result, and the order of the
// additions is the same in every lane: xor distances 1 and 2, mirrored halves of 8 and 16 lanes, then rows of 16 and halves.
template <int G, typename Op>
__device__ __forceinline__ float lanes_reduce(float x)
{
#define CONVFWD_DPP(ctrl) __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), ctrl, 0xF, 0xF, false))
    if constexpr (G >= 2) x = Op::of(x, CONVFWD_DPP(0xB1));   // quad_perm [1,0,3,2]
    if constexpr (G >= 4) x = Op::of(x, CONVFWD_DPP(0x4E));   // quad_perm [2,3,0,1]
    if constexpr (G >= 8) x = Op::of(x, CONVFWD_DPP(0x141));  // row_half_mirror: the other quad of 8 lanes
    if constexpr (G >= 16) x = Op::of(x, CONVFWD_DPP(0x140)); // row_mirror: the other half of 16 lanes
#undef CONVFWD_DPP
    if constexpr (G >= 32) {
        const uint32_t u = __builtin_bit_cast(uint32_t, x);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = Op::of(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
    }
    if constexpr (G >= 64) {
        const uint32_t u = __builtin_bit_cast(uint32_t, x);
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        x = Op::of(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
    }
    return x;
}

// The sum over the lanes of a wave that are G apart (G = 8, 16 or 32); every lane gets it.
template <int G>
__device__ __forceinline__ float across_rows(float x)
{
    if constexpr (G <= 8) x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x128, 0xF, 0xF, false));  // row_ror 8
    if constexpr (G <= 16) {
        const uint32_t u = __builtin_bit_cast(uint32_t, x);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
    }
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// ... over a workgroup of W waves; `lds` holds W floats and is free again after the next barrier of the caller's.
template <int W, typename Op>
__device__ __forceinline__ float block_reduce(float x, float* lds)
{
    x = lanes_reduce<64, Op>(x);
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) lds[wave] = x;
        __syncthreads();
        x = lds[0];
#pragma unroll
        for (int i = 1; i < W; ++i) x = Op::of(x, lds[i]);
    }
    return x;
}

}  // namespace convfwd
