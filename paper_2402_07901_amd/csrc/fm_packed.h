// Shared pieces of the packed attention (fm_packed_fwd.hip, fm_packed_bwd.hip):
// sequences one after the other in [T, H, D] rows, query heads sharing key heads.
//
// Rows are the (token, query head) pairs of a key head, token by token; a
// sequence's rows of one key head form the "row" side, its keys the "key" side.
// A wave holds 32 rows or keys of one side as its columns, in registers, and
// walks over the other side 32 at a time, 64 (float32, D = 128: 32) to an LDS
// tile for a workgroup's four waves:
//   S = X own^T          32x32 scores: X the tile, own the columns
//   acc += X^T w         w made of S, element for element where S left it
// (lane = 32 hh + c32; accumulator register i: column c32, row 8 (i/4) + 4 hh + i%4.)
//
// bf16 calls work on fp16: q^ and k^ (|x| <= sqrt D) have three bits more than
// bf16; a row of v (dO) is an exact fp16 row times a power of two of its own,
// which leaves all but what is 2^-17 of the row's largest.  The powers go into
// the weights, relative to the largest so far: a wave that meets a larger one scales
// its sums down.  Where every column sees the whole tile, one power serves the wave;
// in the tiles that the mask cuts every column (lane) has its own, of what it sees: a
// row keeps its bits beside later tokens of any size (O and dq; dk and dv: of dO's rows up
// to 2^40 larger).  32x32x16 MFMA: one 16-byte LDS
// read per lane and 16 channels for scores, the transposing read for X^T.
// float32 calls: float32 MFMA (32x32x2), operands in full, no powers.
//
// Tiles come straight from the planes that the prep kernel writes (k^, v; backward
// also q^ and dO, [key head][row][D]) into LDS, double buffered.  LDS rows have
// no padding: piece c of row r (16 bytes) lies at c ^ swizzle(r), which puts 8
// consecutive rows' piece c, and pieces c, c + 1 of 4 consecutive rows, on distinct
// banks.  (Over 16 rows instead, a quarter fewer conflicts: the same time in the
// forward, 5 to 10 % longer in the backward, whose addresses take more registers.)
//
// What is not finite.  A tile that is contracted (X^T w) holds zeros in the place of
// infinities and NaN, so that weight 0 of a row that does not see one leaves it out;
// the rows that do get it at the end, from the marks that the prep kernel leaves
// (forward: v; backward: dO), or through G and delta, which are not finite then.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fm_common.h"
#include "fm_internal.h"
#include "fm_pairs_rows.h"
#include "fm_serve.h"

namespace fm {
namespace packed {

using pr::f16v;
using pr::h4;
using pr::h8;
typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256;
constexpr int WAIT_LOADS = 0x0f70;         // vmcnt(0), the other counters at their most
constexpr int NO_POWER = -1000;            // of a row of zeros
constexpr int ROOM = 8;                    // D values of up to 2^128 add up to less than 2^(128 + ROOM)

template <typename T> struct plane_of { typedef float type; };
template <> struct plane_of<bf16_t> { typedef _Float16 type; };

__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <int C> __device__ __forceinline__ int swizzle(int r)
{
    if constexpr (C >= 8) return (r & 3) << 1 | (r >> 2 & 1);
    else if constexpr (C == 4) return (r >> 1 & 1) << 1 | (r >> 2 & 1);   // two rows to a line of banks
    else return r >> 2 & 1;
}

// 16 bytes of every lane from global memory to LDS at `to` + 16 lane.
__device__ __forceinline__ void to_lds(const void *from, void *to)
{
    typedef const uint32_t __attribute__((address_space(1))) *gp;
    typedef uint32_t __attribute__((address_space(3))) *lp;
    __builtin_amdgcn_global_load_lds((gp)from, (lp)to, 16, 0, 0);
}

// Largest over a wave's lanes.
__device__ __forceinline__ int wave_max(int x)
{
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x140, 0xF, 0xF, true));
    const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
    x = max((int)a[0], (int)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
    return scalar(max((int)b[0], (int)b[1]));
}

__device__ __forceinline__ int wave_min(int x) { return -wave_max(-x); }

// The largest x of the lanes 0 .. i, or i .. N - 1, of every N; none: NO_POWER.
template <int N> __device__ __forceinline__ int max_to(int x, int lane, int i)
{
#pragma unroll
    for (int o = 1; o < N; o *= 2) {
        const int y = __shfl_up(x, o, N);
        x = lane % N >= o ? max(x, y) : x;
    }
    const int y = __shfl(x, min(max(i, 0), N - 1), N);
    return i < 0 ? NO_POWER : y;
}
template <int N> __device__ __forceinline__ int max_from(int x, int lane, int i)
{
#pragma unroll
    for (int o = 1; o < N; o *= 2) {
        const int y = __shfl_down(x, o, N);
        x = lane % N + o < N ? max(x, y) : x;
    }
    const int y = __shfl(x, min(max(i, 0), N - 1), N);
    return i >= N ? NO_POWER : y;
}

// What a wave does with rows 32 kb .. 32 kb + 31 of a tile t.
template <typename E, int D> struct Ops;

template <int D> struct Ops<_Float16, D> {
    typedef _Float16 E;
    static constexpr int C = D / 8, KS = D / 16, DT = D < 32 ? 1 : D / 32, TILE = 64;
    static constexpr bool POWERS = true;
    struct Own { u4 x[KS]; };
    struct Turned { u4 x[2][DT]; };

    static __device__ __forceinline__ void own(Own &o, const E *row, int hh)
    {
#pragma unroll
        for (int k = 0; k < KS; ++k) o.x[k] = *(const u4 *)(row + 16 * k + 8 * hh);
    }
    static __device__ __forceinline__ f16v scores(const u4 *t, int kb, int hh, int c32, const Own &o)
    {
        u4 x[KS];
#pragma unroll
        for (int i = 0; i < KS; ++i) x[i] = t[(32 * kb + c32) * C + ((2 * i + hh) ^ swizzle<C>(c32))];
        f16v s = f16v{};
#pragma unroll
        for (int i = 0; i < KS; ++i)
            s = pr::mma(__builtin_bit_cast(h8, x[i]), __builtin_bit_cast(h8, o.x[i]), s);
        return s;
    }
    // Two blocks' scores, product after product in turn (a chain of products into one
    // sum waits for each).
    static __device__ __forceinline__ void scores2(const u4 *t0, int kb0, const Own &o0, f16v &s0, const u4 *t1, int kb1,
                                                   const Own &o1, f16v &s1, int hh, int c32)
    {
        u4 x0[KS], x1[KS];
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            x0[i] = t0[(32 * kb0 + c32) * C + ((2 * i + hh) ^ swizzle<C>(c32))];
            x1[i] = t1[(32 * kb1 + c32) * C + ((2 * i + hh) ^ swizzle<C>(c32))];
        }
        s0 = s1 = f16v{};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            s0 = pr::mma(__builtin_bit_cast(h8, x0[i]), __builtin_bit_cast(h8, o0.x[i]), s0);
            s1 = pr::mma(__builtin_bit_cast(h8, x1[i]), __builtin_bit_cast(h8, o1.x[i]), s1);
        }
    }
    // X^T: rows {4 hh .. + 3, 8 + 4 hh .. + 3} of 16, channel c32 of 32 (D = 16: the
    // upper 16 repeat the lower)
    static __device__ __forceinline__ void turn(Turned &a, const u4 *t, int kb, int lane)
    {
        const s4 *v = (const s4 *)t;
        const int j = lane >> 2 & 3, hh = lane >> 5;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                typedef s4 __attribute__((address_space(3))) *lp;
                const int r = 32 * kb + 16 * m + 4 * hh + j;
                const int c = 4 * d + (D < 32 ? 0 : 2 * (lane >> 4 & 1)) + (lane >> 1 & 1);
                const int at = 2 * (r * C + (c ^ swizzle<C>(4 * hh + j))) + (lane & 1);
                const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(v + at));
                const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(v + at + 2 * 8 * C));
                const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
                a.x[m][d] = u4{l.x, l.y, h.x, h.y};
            }
        }
    }
    static __device__ __forceinline__ void add(f16v *acc, const Turned &a, const pr::h2 *w)
    {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            h8 b;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                b[2 * i] = w[4 * m + i][0];
                b[2 * i + 1] = w[4 * m + i][1];
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = pr::mma(__builtin_bit_cast(h8, a.x[m][d]), b, acc[d]);
        }
    }
    static __device__ __forceinline__ void add(f16v *acc, const Turned &a, const float *w)
    {
        pr::h2 h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = pr::cvt2(w[2 * i], w[2 * i + 1]);
        add(acc, a, h);
    }
    // the channel of register i of accumulator d, the first of 4 neighbours if i % 4 == 0
    static __device__ __forceinline__ int channel(int d, int i, int hh) { return 32 * d + 8 * (i / 4) + 4 * hh + i % 4; }
};

template <int D> struct Ops<float, D> {
    typedef float E;
    static constexpr int C = D / 4, DT = D < 32 ? 1 : D / 32, TILE = D == 128 ? 32 : 64;
    static constexpr bool POWERS = false;
    struct Own { f4 x[D / 8]; };
    struct Turned { float x[16][DT]; };

    // the lanes of half hh hold channels hh D/2 .. (hh + 1) D/2
    static __device__ __forceinline__ void own(Own &o, const E *row, int hh)
    {
#pragma unroll
        for (int j = 0; j < C / 2; ++j) o.x[j] = *(const f4 *)(row + hh * (D / 2) + 4 * j);
    }
    static __device__ __forceinline__ f16v scores(const u4 *t, int kb, int hh, int c32, const Own &o)
    {
        f16v s = f16v{};
#pragma unroll
        for (int j = 0; j < C / 2; ++j) {
            const f4 x = __builtin_bit_cast(f4, t[(32 * kb + c32) * C + ((hh * (C / 2) + j) ^ swizzle<C>(c32))]);
#pragma unroll
            for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], o.x[j][i], s, 0, 0, 0);
        }
        return s;
    }
    static __device__ __forceinline__ void scores2(const u4 *t0, int kb0, const Own &o0, f16v &s0, const u4 *t1, int kb1,
                                                   const Own &o1, f16v &s1, int hh, int c32)
    {
        s0 = scores(t0, kb0, hh, c32, o0);
        s1 = scores(t1, kb1, hh, c32, o1);
    }
    // rows 8 (i/4) + 4 hh + i%4, DT neighbouring channels from c32 DT on (D = 16: the
    // upper lanes repeat the lower)
    static __device__ __forceinline__ void turn(Turned &a, const u4 *t, int kb, int lane)
    {
        const int hh = lane >> 5, ch = (lane & (D < 32 ? 15 : 31)) * DT;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 32 * kb + 8 * (i / 4) + 4 * hh + i % 4;
            const float *v = (const float *)(t + r * C + ((ch / 4) ^ swizzle<C>(r))) + ch % 4;
#pragma unroll
            for (int d = 0; d < DT; ++d) a.x[i][d] = v[d];
        }
    }
    static __device__ __forceinline__ void add(f16v *acc, const Turned &a, const float *w)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[i][d], w[i], acc[d], 0, 0, 0);
    }
    static __device__ __forceinline__ int channel(int d, int i, int hh) { return (8 * (i / 4) + 4 * hh + i % 4) * DT + d; }
};

// The infinities and NaN of marked rows to the columns that see them.  marked(r): is
// row r; begin a multiple of 64; from(r): its channels; sees(r): the lane's column.
template <typename T, int D, typename M, typename F, typename S>
__device__ __forceinline__ void add_odd(f16v *acc, int begin, int end, int lane, M marked, F from, S sees)
{
    using O = Ops<typename plane_of<T>::type, D>;
#pragma unroll 1
    for (int r0 = begin; r0 < end; r0 += 64) {
        uint64_t odd = __ballot(r0 + lane < end && marked(r0 + lane));
#pragma unroll 1
        while (odd) {
            const int r = r0 + __builtin_ctzll(odd);
            odd &= odd - 1;
            const T *row = from(r);
            const bool see = sees(r);
#pragma unroll
            for (int d = 0; d < O::DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int ch = O::channel(d, i, lane >> 5);
                    if (D < 32 && ch >= D) continue;
                    const float x = io<T>::ld(row, ch);
                    if (see && !(fabsf(x) <= 3.4028235e38f)) acc[d][i] += x;
                }
        }
    }
}

// What a workgroup takes: tokens [t0, t0 + len) of a sequence, its first column
// (a row or a key), and what it makes of its columns.  len 0: nothing to do.
enum Role { ROWS = 0, KEYS = 1, DK = 2, DV = 3 };   // O or dq; dk and dv; one of them
struct Place {
    int t0, len, first, role;
};
__device__ __forceinline__ Place scalar(Place p) { return Place{scalar(p.t0), scalar(p.len), scalar(p.first), scalar(p.role)}; }

// The columns of sequences whose tokens have `per` of them each, `cols` to a place:
// sequence s has the places floor(starts[s] per / cols) + s and on, enough for it and
// no other's.
inline long long places(int S, int T, int per, int cols) { return (long long)T * per / cols + S; }

__device__ __forceinline__ Place place_of(const int32_t *starts, int S, int T, int per, int cols, int idx)
{
    const auto at = [&](int s) { return (long long)min(max(starts[s], 0), T) * per / cols + s; };
    int lo = 0, hi = S - 1;   // the last sequence that begins at idx or before
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (at(mid) <= idx) lo = mid;
        else hi = mid - 1;
    }
    const long long first = (idx - at(lo)) * cols;
    Place p = {min(max(starts[lo], 0), T), 0, 0, 0};
    const int len = min(max(starts[lo + 1], p.t0), T) - p.t0;
    if (first >= 0 && first < (long long)len * per) {
        p.len = len;
        p.first = (int)first;
    }
    return p;
}

// Loads tile rows r0 .. r0 + TILE - 1 of two planes (rows past `last` repeat it)
// into LDS: the loads of a wave are every fourth.  A lane's place in a whole tile
// does not change: scalar base, 32-bit offset.
template <typename E, int D, int TILE>
__device__ __forceinline__ void load_tiles(const E *x, const E *y, int r0, int last, u4 *xt, u4 *yt, int wave, int lane)
{
    using O = Ops<E, D>;
    constexpr int C = O::C, LR = 64 / C, N = TILE / LR;   // rows of a load, loads of a tile
    const bool in = r0 + TILE - 1 <= last;
    const char *const xb = (const char *)(x + (size_t)r0 * D), *const yb = (const char *)(y + (size_t)r0 * D);
#pragma unroll
    for (int i = 0; i < (2 * N + 3) / 4; ++i) {
        const int n = wave + 4 * i;
        if (2 * N % 4 && n >= 2 * N) break;
        const int l0 = n % N * LR, r = l0 + lane / C;
        const int at = in ? r : min(r, last - r0);   // last >= r0
        const uint32_t off = (uint32_t)(at * D * (int)sizeof(E) + 16 * (lane % C ^ swizzle<C>(r)));
        to_lds((n < N ? xb : yb) + off, (n < N ? xt : yt) + l0 * C);
    }
}

// Walks over the tiles of rows [begin, end) of two planes: tile r0 is worked on while
// the next one is on its way.  The tiles of [begin2, end2) go to `fast`, the ones before
// and after to `masked`; begin2 and end2 are whole pairs of tiles from begin, or the end.  Four LDS arrays, restrict: a load
// into one buffer need not be waited for before the other is read.
template <typename E, int D, int TILE, typename F, typename M>
__device__ __forceinline__ void walk(const E *x, const E *y, int begin, int begin2, int end2, int end, int last,
                                     u4 *__restrict__ x0, u4 *__restrict__ x1, u4 *__restrict__ y0, u4 *__restrict__ y1,
                                     int wave, int lane, F fast, M masked)
{
    if (begin < end) load_tiles<E, D, TILE>(x, y, begin, last, x0, y0, wave, lane);
    __builtin_amdgcn_s_waitcnt(WAIT_LOADS);
    __syncthreads();
    if (begin + TILE < end) load_tiles<E, D, TILE>(x, y, begin + TILE, last, x1, y1, wave, lane);
    // the next tile is there, and this one's buffer is free
    const auto turn = [&](int r0, u4 *xt, u4 *yt) {
        __builtin_amdgcn_s_waitcnt(WAIT_LOADS);
        __syncthreads();
        if (r0 + 2 * TILE < end) load_tiles<E, D, TILE>(x, y, r0 + 2 * TILE, last, xt, yt, wave, lane);
    };
    const auto pairs = [&](int r0, int to, auto &compute) {
        for (; r0 < to; r0 += 2 * TILE) {
            compute(x0, y0, r0);
            turn(r0, x0, y0);
            if (r0 + TILE < end) {
                compute(x1, y1, r0 + TILE);
                turn(r0 + TILE, x1, y1);
            }
        }
    };
    pairs(begin, begin2, masked);
    pairs(begin2, end2, fast);
    pairs(end2, end, masked);
}

// How a workgroup's four waves share its work: WK = 1, each 32 columns of 128 and all
// tiles; WK = 4, the same 32 columns and every fourth block of 32 rows, their sums added
// in LDS at the end.  Calls that would leave CUs idle with 128 columns take 32: one
// prompt of 777 tokens, 12 heads of 64: 84 workgroups, 300 of a quarter of the steps.
template <typename E, int D, int WK> struct Cut {
    static constexpr int COLS = WK == 1 ? 128 : 32;
    static constexpr int TILE = WK == 1 ? Ops<E, D>::TILE : 128;
    static constexpr int MINE = WK == 1 ? TILE : 32;    // of a tile, a wave's
    // two buffers of two tiles fit a CU's LDS
    static constexpr bool FITS = WK == 1 || 4 * TILE * D * (int)sizeof(E) <= 128 * 1024;
    static_assert(TILE * D * (int)sizeof(E) >= Ops<E, D>::DT * 16 * 64 * 4 || WK == 1, "an array for a wave's sums");
};

// Adds the waves' sums (times 2^power of each column) in LDS, one array per wave (a tile's:
// at least 4 KB for 32 channels); power becomes that of the sum.  The caller has made
// sure that the arrays are free, and puts a barrier between.
template <int DT>
__device__ __forceinline__ void join_put(f16v *acc, int &power, int (*powers)[64], u4 *mine, int wave, int lane)
{
    powers[wave][lane] = power;
    __syncthreads();
    const int most = max(max(powers[0][lane], powers[1][lane]), max(powers[2][lane], powers[3][lane]));
    const float f = __builtin_ldexpf(1.0f, max(power - most, -300));
    power = most;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) ((float *)mine)[(16 * d + i) * 64 + lane] = acc[d][i] * f;
}
template <int DT>
__device__ __forceinline__ void join_get(f16v *acc, const u4 *a, const u4 *b, const u4 *c, const u4 *e, int lane)
{
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int j = (16 * d + i) * 64 + lane;
            acc[d][i] = (((const float *)a)[j] + ((const float *)b)[j]) + (((const float *)c)[j] + ((const float *)e)[j]);
        }
}

// Four neighbouring values (n of them where fewer) of a row.
template <int N> __device__ __forceinline__ void put(float *p, const float *f)
{
    if constexpr (N == 4) *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
    else if constexpr (N == 2) *(float2 *)p = make_float2(f[0], f[1]);
    else *p = *f;
}
template <int N> __device__ __forceinline__ void put(bf16_t *p, const float *f)
{
    static_assert(N == 4, "a register quad");
    *(uint2 *)p = make_uint2(mx::pack_bf16x2(f[0], f[1]), mx::pack_bf16x2(f[2], f[3]));
}
// Stores a column's channels as a row.
template <typename T, int D>
__device__ __forceinline__ void store_row(T *row, const f16v *acc, int hh)
{
    using O = Ops<typename plane_of<T>::type, D>;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int N = F32 ? O::DT : 4;
#pragma unroll
    for (int n = 0; n < 16 * O::DT / N; ++n) {
        // bf16: a register quad of one accumulator; float32: a register of every one
        const int d0 = F32 ? 0 : n / 4, i0 = F32 ? n : n % 4 * 4, ch = O::channel(d0, i0, hh);
        if (D < 32 && ch >= D) continue;
        float f[N];
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = F32 ? acc[j][i0] : acc[d0][i0 + j];
        put<N>(row + ch, f);
    }
}

// What the prep kernel leaves (workspace): the places, and per key (key head, token)
// and, for the backward, per row (key head, token, head in its group):
struct RowInfo {
    float m;        // 1 / G times 2^a is m 2^e, a the power of dO; float32: 1 / G
    int e;          // NO_POWER: dO is zeros
    float delta;    // dO.O 2^-(a + ROOM); float32: dO.O
    int ed;         // twice the least power above it, + 1 if dO has what is not finite
};
template <typename E> struct Planes {
    E *kh, *vh, *qh, *oh;
    int *b;              // twice the power of v, + 1 if v has what is not finite
    float *rk, *rq;      // 1 / std of k and q
    RowInfo *info;
    Place *places;
    int n_places, sorted;
    int split;           // dk and dv by workgroups of their own
    int cols;            // columns of a workgroup
};
// At D = 128, bf16, the sums of dk and dv leave no registers for two waves on a SIMD;
// the scores made twice cost less (a seventh more products).
constexpr bool split_keys(int D, bool bf16) { return bf16 && D == 128; }
// Scores of a whole tile before its weights, where registers allow it.
template <typename E, int D> constexpr bool ahead() { return D < 128; }
template <typename E> Planes<E> planes_at(void *ws, const PackedArgs &a, int D, int backward);
// Whether a call takes 32 columns to a workgroup.
bool small_call(int S, int T, int Hq, int Hkv, int D, int is_bf16, int backward);
template <typename T, typename E>
hipError_t prep(const PackedArgs &a, const Planes<E> &p, int D, int backward, hipStream_t st);

}  // namespace packed
}  // namespace fm
