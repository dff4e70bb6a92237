// A row of D channels as the row kernels hold it (fm_rows.hip): D / 16 lanes,
// 16 channels each, as two runs of 8 that hold both sides of 8 rotation pairs.
//
// Rotation of the first `rot` channels (rot a multiple of 16), by pairs (a, b):
//     a' = a cos - b sin,  b' = b cos + a sin
// with pair j = (j, j + rot/2), or (2j, 2j + 1) when interleaved.  Lane c of a
// row holds the pairs 8c .. 8c + 7, so no lane needs another's channels; the
// lanes past rot/16 hold 16 unrotated channels each.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fm_common.h"
#include "fm_serve.h"

namespace fm {
namespace rows {

__device__ __forceinline__ void ld8(const float *p, float *x)
{
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

__device__ __forceinline__ void ld8(const bf16_t *p, float *x)
{
    const uint4 u = *(const uint4 *)p;
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ void st8(float *p, const float *x)
{
    *(float4 *)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4 *)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// Two floats -> two bf16 (round to nearest even) packed low-first.
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    typedef float fl2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(fl2{a, b}, bf2));
}

__device__ __forceinline__ void st8(bf16_t *p, const float *x)
{
    *(uint4 *)p = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
}

// Sum over the L lanes of a row (L in 1, 2, 4, 8, aligned) with DPP: swap
// neighbours, swap pairs, mirror the two quads of each half row.
template <int L> __device__ __forceinline__ float row_sum(float x)
{
    if constexpr (L >= 2)
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xF, 0xF, true));
    if constexpr (L >= 4)
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xF, 0xF, true));
    if constexpr (L >= 8)
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xF, 0xF, true));
    return x;
}

// The largest of the lanes' values, likewise.
template <int L> __device__ __forceinline__ uint32_t row_max(uint32_t x)
{
    if constexpr (L >= 2) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));
    if constexpr (L >= 4) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));
    if constexpr (L >= 8) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));
    return x;
}

// A lane's place in its row: where its two runs of 8 channels start, and
// whether they are rotated.
struct Place {
    int a, b;
    bool turned;
};

__device__ __forceinline__ Place place_of(int c, const Rope &r)
{
    const int half = r.half;
    if (r.interleaved || 8 * c >= half) return Place{16 * c, 16 * c + 8, 8 * c < half};
    return Place{8 * c, half + 8 * c, true};
}

// cos and sin of the lane's 8 pairs for token t.  A position outside the
// table has no rotation: its rows come out as NaN rather than from memory
// past the table.
__device__ __forceinline__ void angles(const Rope &r, long long t, int c, float *cs, float *sn)
{
    const int j = 8 * c;
    if (r.axes == 1) {
        const int p = r.pos[t];
        const bool ok = (unsigned)p < (unsigned)r.table_rows;
        const size_t at = (size_t)(ok ? p : 0) * r.half + j;
        ld8(r.cos + at, cs);
        ld8(r.sin + at, sn);
        if (!ok) {
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[i] = sn[i] = __builtin_nanf("");
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int axis = (j + i >= r.end[0]) + (j + i >= r.end[1]) + (j + i >= r.end[2]);
        const int p = r.pos[t * r.axes + axis];
        const bool ok = (unsigned)p < (unsigned)r.table_rows;
        const size_t at = (size_t)(ok ? p : 0) * r.half + j + i;
        cs[i] = ok ? r.cos[at] : __builtin_nanf("");
        sn[i] = ok ? r.sin[at] : __builtin_nanf("");
    }
}

// The rotation of a lane's 16 channels; BACK rotates the other way (its
// transpose, which carries gradients).
template <bool BACK>
__device__ __forceinline__ void turn(float *x, const float *cs, const float *sn, bool interleaved)
{
    // the pair's two channels: i and i + 8, or 2 i and 2 i + 1
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = BACK ? -sn[i] : sn[i], a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = fmaf(a, cs[i], -(b * s));
            x[2 * i + 1] = fmaf(b, cs[i], a * s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = BACK ? -sn[i] : sn[i], a = x[i], b = x[i + 8];
            x[i] = fmaf(a, cs[i], -(b * s));
            x[i + 8] = fmaf(b, cs[i], a * s);
        }
    }
}

}  // namespace rows
}  // namespace fm
