// Paged attention of many rows of a sequence (chunks of prompts).
//
// MFMA bounds it, so keys and values are staged in LDS for a workgroup's 128
// rows, 64 keys at a time (float32 at D = 128: 32), and each of its four waves
// works on 32 rows with 32x32 tiles.  bf16, 32x32x16:
//   S^T = K Q^T    A: 32 keys (one 16-byte LDS read per lane and 16 channels),
//                  B: q^ of 32 rows, in registers throughout
//   O^T += V^T W^T B: the weights, which the accumulator layout of S^T holds
//                  where B wants them if a 16-key step takes keys
//                  {4h..4h+3, 8+4h..8+4h+3} for the lanes of half h; A: the
//                  same keys of 32 channels, through the transposing LDS read
// (lane = 32 h + c32; accumulator register i: column c32, row 8 (i/4) + 4 h + i%4).
// float32, 32x32x2: the lanes of half h hold channels h D/2 .. (h + 1) D/2 of
// K and Q, 16 bytes at a time; the weights of accumulator register i are B of
// the step with keys 8 (i/4) + i%4 and 4 more, and with channel c32 D/32 + d in
// row c32 of A for product d a lane reads D/32 neighbouring channels of a key.
// The next keys go straight to the other LDS buffer (global_load_lds) while
// these are worked on.  Registers: two waves on a SIMD, from two workgroups,
// whose products and weights overlap.  64 rows per wave read LDS half as often
// but leave one wave on a SIMD at D = 128 (10 % slower).
//
// LDS rows have no padding; the 16-byte piece c of row r lies
// at piece c ^ swizzle(r), which puts 8 consecutive rows' piece c (score
// operands) and pieces c, c + 1 of 4 consecutive rows (value operands) on
// distinct banks.
//
// In bf16 the weights enter as two bf16 parts, 16 bits of each: rounded to one
// they would add as much error again as the output's own rounding (2.5e-3
// against 1.6e-3 of the output's size on short rows), for half as many MFMA
// again.  Eight chunks of 2048 rows over 8192 keys, 32 heads to 8, D = 128:
// 2.53 to 2.62 ms, 735 to 760 TFLOP/s of the formula's products and 1.10 to
// 1.14 PFLOP/s of those executed, where a large matrix product reaches 1.21;
// MFMA busy 58 % at the 1.9 GHz that this load leaves.  D = 64: 660 to 700.
// float32, 4096 keys: 105 of 154 TFLOP/s at D = 128, 113 at D = 64, MFMA busy
// 78 %.
#include <hip/hip_runtime.h>

#include "fm_internal.h"
#include "fm_paged.h"
#include "fm_rows.h"
#include "fm_serve.h"

namespace fm {
namespace {

using namespace paged;

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256;
constexpr int WAIT_LOADS = 0x0f70;   // vmcnt(0), the other counters at their most

// C: 16-byte pieces of a row
template <int C> __device__ __forceinline__ int swizzle(int r)
{
    if constexpr (C >= 8) return (r & 3) << 1 | (r >> 2 & 1);
    else return (r >> 1 & 1) << 1 | (r >> 2 & 1);   // two rows to a line of banks
}

__device__ __forceinline__ f16v mma(u4 a, u4 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

// Sum of a lane's and its partner's (lane ^ 32) values, in both.
__device__ __forceinline__ float halves_sum(float x)
{
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// 16 bytes of every lane from global memory to LDS at `to` + 16 lane.
__device__ __forceinline__ void to_lds(const void *from, void *to)
{
    typedef const uint32_t __attribute__((address_space(1))) *gp;
    typedef uint32_t __attribute__((address_space(3))) *lp;
    __builtin_amdgcn_global_load_lds((gp)from, (lp)to, 16, 0, 0);
}

// What a wave does with 32 keys `kb` of a buffer: scores of its 32 rows, weights
// from scores (and their sum: rounded where they are), values under them.
template <typename T, int D> struct Wave;

template <int D> struct Wave<bf16_t, D> {
    static constexpr int C = D / 8, KC = D / 16, DT = D / 32;
    u4 q[KC], va[2][DT];

    __device__ __forceinline__ void load_q(const bf16_t *p, int hh)
    {
#pragma unroll
        for (int k = 0; k < KC; ++k) q[k] = *(const u4 *)(p + 16 * k + 8 * hh);
    }
    __device__ __forceinline__ f16v scores(const u4 *kl, int kb, int hh, int c32) const
    {
        u4 k[KC];
#pragma unroll
        for (int i = 0; i < KC; ++i) k[i] = kl[(32 * kb + c32) * C + ((2 * i + hh) ^ swizzle<C>(c32))];
        f16v x = f16v{};
#pragma unroll
        for (int i = 0; i < KC; ++i) x = mma(k[i], q[i], x);
        return x;
    }
    // The value operands are read ahead of the weights.
    __device__ __forceinline__ void read(const u4 *vl, int kb, int lane)
    {
        const s4 *v = (const s4 *)vl;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                typedef s4 __attribute__((address_space(3))) *lp;
                const int j = lane >> 2 & 3, hh = lane >> 5, r = 32 * kb + 16 * m + 4 * hh + j;
                const int c = 4 * d + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
                const int at = 2 * (r * C + (c ^ swizzle<C>(4 * hh + j))) + (lane & 1);
                const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(v + at));
                const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(v + at + 2 * 8 * C));
                const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
                va[m][d] = u4{l.x, l.y, h.x, h.y};
            }
        }
    }
    __device__ __forceinline__ void add(f16v *acc, float &g, const f16v &w, const u4 *, int, int, int) const
    {
        u4 hi[2], lo[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = w[2 * i], y = w[2 * i + 1];
            g += x + y;
            // hi: the upper 16 bits; lo: the rest, of the same sign and never 0
            // (x | 1), so that an infinite value stays one under both
            hi[i / 4][i % 4] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
            lo[i / 4][i % 4] = rows::pack2(rest(x), rest(y));
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = mma(va[m][d], hi[m], acc[d]);
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = mma(va[m][d], lo[m], acc[d]);
        }
    }
    static __device__ __forceinline__ float rest(float x)
    {
        return __uint_as_float(__float_as_uint(x) | 1u) - __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    }
    // channel of register i of accumulator d
    static __device__ __forceinline__ int channel(int d, int i, int hh) { return 32 * d + 8 * (i / 4) + 4 * hh + i % 4; }
};

template <int D> struct Wave<float, D> {
    static constexpr int C = D / 4, DT = D / 32;
    f4 q[D / 8];

    __device__ __forceinline__ void load_q(const float *p, int hh)
    {
#pragma unroll
        for (int j = 0; j < C / 2; ++j) q[j] = *(const f4 *)(p + hh * (D / 2) + 4 * j);
    }
    __device__ __forceinline__ f16v scores(const u4 *kl, int kb, int hh, int c32) const
    {
        f16v x = f16v{};
#pragma unroll
        for (int j = 0; j < C / 2; ++j) {
            const f4 k = __builtin_bit_cast(f4, kl[(32 * kb + c32) * C + ((hh * (C / 2) + j) ^ swizzle<C>(c32))]);
#pragma unroll
            for (int i = 0; i < 4; ++i) x = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i], q[j][i], x, 0, 0, 0);
        }
        return x;
    }
    __device__ __forceinline__ void read(const u4 *, int, int) {}
    __device__ __forceinline__ void add(f16v *acc, float &g, const f16v &w, const u4 *vl, int kb, int hh, int c32) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 32 * kb + 8 * (i / 4) + 4 * hh + i % 4, ch = c32 * DT;
            const float *v = (const float *)(vl + r * C + ((ch / 4) ^ swizzle<C>(r))) + ch % 4;
            g += w[i];
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[d], w[i], acc[d], 0, 0, 0);
        }
    }
    static __device__ __forceinline__ int channel(int d, int i, int hh) { return (8 * (i / 4) + 4 * hh + i % 4) * DT + d; }
};

// N neighbouring channels
template <int N> __device__ __forceinline__ void put(float *p, const float *f)
{
    if constexpr (N == 4) *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
    else if constexpr (N == 2) *(float2 *)p = make_float2(f[0], f[1]);
    else *p = *f;
}
template <int N> __device__ __forceinline__ void put(bf16_t *p, const float *f)
{
    static_assert(N == 4, "a register quad");
    *(uint2 *)p = make_uint2(rows::pack2(f[0], f[1]), rows::pack2(f[2], f[3]));
}

__device__ __forceinline__ bool odd_bits(bf16_t v) { return (v & 0x7f80) == 0x7f80; }
__device__ __forceinline__ bool odd_bits(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }
// one among 16 bytes of them
template <typename T> __device__ __forceinline__ bool odd_bits(u4 x)
{
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        odd |= odd_bits(__uint_as_float(x[i]));   // bf16: the upper one
        if constexpr (sizeof(T) == 2) odd |= odd_bits((bf16_t)x[i]);
    }
    return odd;
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS, sizeof(T) == 2 && D == 64 ? 3 : 2) void chunk_kernel(PagedArgs a, PagedPlan plan, int pieces, float *part)
{
    constexpr int ROWS = CHUNK_ROWS, WR = ROWS / 4;   // rows of a workgroup, of a wave
    using W = Wave<T, D>;
    constexpr int C = W::C, DT = W::DT, P = 16 / sizeof(T);   // 16-byte pieces of a row, channels of a piece
    constexpr int KB = C > 16 ? 32 : 64;           // keys of an LDS buffer: two workgroups to a CU
    constexpr int LR = 64 / C;                     // rows that a wave's load covers
    constexpr int LN = KB / LR / 4;                // loads of a wave, of keys and of values
    // two buffers
    __shared__ u4 keys0[KB * C], keys1[KB * C], values0[KB * C], values1[KB * C];
    // channels of a row that met +infinity, -infinity (both: NaN) where not
    // every row sees the key
    __shared__ uint32_t flags[2][ROWS][DT];

    // Row tiles of one (sequence, key head, split) read the same keys, so every
    // `pieces`th of them go to the same XCD (workgroups are dealt out to the 8
    // XCDs in turn).  Late row tiles see the most keys and start first.
    const int in_piece = (plan.tiles + pieces - 1) / pieces;
    const int turn = blockIdx.x / 8 / in_piece, piece = turn * 8 + (blockIdx.x + turn) % 8;
    const int row_tile = plan.tiles - 1 - (piece % pieces + pieces * (blockIdx.x / 8 % in_piece));
    const int split = piece / pieces % plan.splits, pair = piece / pieces / plan.splits;
    if (pair >= a.S * a.Hkv || row_tile < 0) return;
    const int head = pair % a.Hkv, s = pair / a.Hkv;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = threadIdx.x % 64, hh = lane / 32, c32 = lane % 32;
    const Seq seq = seq_of(a, s);
    const int rows = seq.count * a.group, page_mask = (1 << a.page_shift) - 1;
    const T *kc = (const T *)a.k + head * a.cache.head, *vc = (const T *)a.v + head * a.cache.head;
    const int32_t *table = a.table + (size_t)s * a.table_cols;

    uint32_t lane_at[LN];   // bytes from a tile's first row to what the lane loads
#pragma unroll
    for (int i = 0; i < LN; ++i) {
        const int r = (wave + 4 * i) * LR + lane / C;
        lane_at[i] = (uint32_t)sizeof(T) * (r % KT * (uint32_t)a.cache.token + P * (lane % C ^ swizzle<C>(r)));
    }

    for (int r0 = row_tile * ROWS; r0 < rows; r0 += plan.tiles * ROWS) {
        const Span sp = scalar(span_of_rows(a, seq, r0, ROWS));
        const int begin = split * plan.chunk;
        const int end = split == plan.splits - 1 ? sp.tiles : min(sp.tiles, begin + plan.chunk);
        if (begin >= sp.tiles && split > 0) continue;   // the join knows
        const int pos0 = seq.len - seq.count;           // position of row 0
        const int first = scalar(pos0 + r0 / a.group), last = sp.end - 1;

        const int row = r0 + wave * WR + c32;           // the lane's own
        const int t = min(row, rows - 1) / a.group, pos = pos0 + t;
        const int q_head = head * a.group + min(row, rows - 1) - t * a.group;
        W wv;
        wv.load_q((const T *)a.q + (seq.t0 + t) * a.q_token + q_head * a.q_head, hh);
        f16v acc[DT];
        float g = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = f16v{};

        bool bad = seq.cut, met_odd = false;
        // Key tiles [whole, whole_end) exist in full and every row sees all their
        // keys; elsewhere keys are clamped and weights masked.
        const int shift = sp.low - sp.sink_tiles;   // from a tile's number here to its own
        const int whole = a.window < sp.end ? max(sp.sink_tiles, (last - a.window) / KT + 1 - shift) : 0;
        const int whole_end = min(end, (first + 1) / KT - shift);
        // Where the key tiles i0 .. i0 + 3 begin in the cache, in lanes 0 .. 3 (a
        // vector load a step ahead: nothing waits for it).
        const auto page_of = [&](int i0) {
            return table[sp.tile(min(i0 + lane % 4, end - 1)) * KT >> a.page_shift];
        };
        const auto tile_of = [&](int i0, int page) {
            if ((unsigned)page >= (unsigned)a.pages) {
                bad = true;
                page = 0;
            }
            const int n0 = sp.tile(min(i0 + lane % 4, end - 1)) * KT;
            return page * a.cache.batch + (n0 & page_mask) * a.cache.token;
        };
        // Loads key tiles i0 .. i0 + 3 into a buffer.  The rows of one load are in
        // one tile, so all but a lane's place in the tile is scalar.
        const auto load = [&](int i0, u4 *kd, u4 *vd, int page) {
            const long long at = tile_of(i0, page);
            const bool all = i0 >= whole && i0 + KB / KT <= whole_end;
#pragma unroll
            for (int i = 0; i < LN; ++i) {
                const int l0 = (wave + 4 * i) * LR, it = l0 / KT;
                const long long from = (long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(at >> 32), it) << 32 |
                                                   (uint32_t)__builtin_amdgcn_readlane((int)at, it));
                uint32_t off = lane_at[i];
                if (!all) {
                    const int n0 = sp.tile(min(i0 + it, end - 1)) * KT, r = l0 + lane / C;
                    off = (uint32_t)sizeof(T) * ((sp.read(n0 + r % KT, n0 + KT - 1) - n0) * (uint32_t)a.cache.token + P * (lane % C ^ swizzle<C>(r)));
                }
                to_lds((const char *)(kc + from) + off, kd + l0 * C);
                to_lds((const char *)(vc + from) + off, vd + l0 * C);
            }
        };
        const auto unseen = [&](int i0) { return i0 < whole || i0 + KB / KT > whole_end; };
        // An infinity or a NaN among values that some row may not see: weight 0
        // would make it NaN there, so it leaves the buffer, and the rows that
        // do see it are marked.  (Looked for 16 bytes at a time: the diagonal
        // and a window's edges are all that a short chunk has.)
        const auto screen = [&](int i0, u4 *vd) {
#pragma unroll
            for (int piece = threadIdx.x; piece < KB * C; piece += THREADS) {
                if (!odd_bits<T>(vd[piece])) continue;
                const int r = piece / C, c = piece % C ^ swizzle<C>(r);
                T *x = (T *)&vd[piece];
#pragma unroll 1
                for (int e = 0; e < P; ++e) {
                    const T v = x[e];
                    if (!odd_bits(v)) continue;
                    x[e] = 0;
                    met_odd = true;
                    if (i0 + r / KT >= end) continue;
                    const int n = sp.tile(i0 + r / KT) * KT + r % KT;
#pragma unroll 1
                    for (int i = 0; i < ROWS && r0 + i < rows; ++i) {
                        const int t = (r0 + i) / a.group;
                        if (!visible(n, pos0 + t, a.window, a.sinks)) continue;
                        bool nan = isnan(io<T>::ld(&v, 0)), neg = io<T>::ld(&v, 0) < 0.f;
                        if (!nan && a.c2 == 0.f) {   // first order: the weight may be negative, or 0
                            const T *qp = (const T *)a.q + (seq.t0 + t) * a.q_token +
                                          (head * a.group + r0 + i - t * a.group) * a.q_head;
                            const int page = min((unsigned)table[n >> a.page_shift], (unsigned)a.pages - 1);
                            const T *kp = kc + page * a.cache.batch + (n & page_mask) * a.cache.token;
                            float dot = 0.f;
#pragma unroll 1
                            for (int d = 0; d < D; ++d) dot = fmaf(io<T>::ld(qp, d), io<T>::ld(kp, d), dot);
                            const float w = fmaf(dot, a.c1, 1.0f);
                            nan = w == 0.f;
                            neg ^= w < 0.f;
                        }
                        const int ch = P * c + e;
                        if (nan || !neg) atomicOr(&flags[0][i][ch / 32], 1u << (ch % 32));
                        if (nan || neg) atomicOr(&flags[1][i][ch / 32], 1u << (ch % 32));
                    }
                }
            }
            __syncthreads();
        };

        for (int i = threadIdx.x; i < 2 * ROWS * DT; i += THREADS) (&flags[0][0][0])[i] = 0;
        // Restrict: a load into one buffer need not be waited for before the
        // other is read.
        const auto walk = [&](u4 *__restrict__ k0, u4 *__restrict__ k1, u4 *__restrict__ v0, u4 *__restrict__ v1) {
            constexpr int STEP = KB / KT;
            // 64 keys from buffers k, v; those after them are on the way to the
            // others (ko, vo), the ones after those come here.
            const auto step = [&](int i0, u4 *k, u4 *v, u4 *vo) {
                const bool all = !unseen(i0);
                const int page = page_of(i0 + 2 * STEP);
#pragma unroll
                for (int kb = 0; kb < KB / 32; ++kb) {
                    f16v x = wv.scores(k, kb, hh, c32);
                    wv.read(v, kb, lane);
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = fmaf(fmaf(x[i], a.c2, a.c1), x[i], 1.0f);
                    if (!all) {
                        // key n0 + e of a tile is seen if e <= lim and (e > lim - window
                        // or it is a first token)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int it = i0 + 2 * kb + j, n0 = sp.tile(min(it, end - 1)) * KT + 4 * hh;
                            const int lim = it < end ? max(pos, -1) - n0 : -1, low = lim - a.window, sinks = a.sinks - n0;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const int e = 8 * (i / 4) + i % 4;
                                if (e > lim || (e <= low && e >= sinks)) x[8 * j + i] = 0.f;
                            }
                        }
                    }
                    wv.add(acc, g, x, v, kb, hh, c32);
                }
                // the next keys are there, and these buffers are free
                __builtin_amdgcn_s_waitcnt(WAIT_LOADS);
                __syncthreads();
                if (i0 + STEP < end && unseen(i0 + STEP)) screen(i0 + STEP, vo);
                if (i0 + 2 * STEP < end) load(i0 + 2 * STEP, k, v, page);
            };
            if (begin < end) load(begin, k0, v0, page_of(begin));
            __builtin_amdgcn_s_waitcnt(WAIT_LOADS);   // q^ too: no wait for it in the loop
            __syncthreads();
            if (begin < end) {
                if (unseen(begin)) screen(begin, v0);
                if (begin + STEP < end) load(begin + STEP, k1, v1, page_of(begin + STEP));
            }
            for (int i0 = begin; i0 < end; i0 += 2 * STEP) {
                step(i0, k0, v0, v1);
                if (i0 + STEP < end) step(i0 + STEP, k1, v1, v0);
            }
        };
        walk(keys0, keys1, values0, values1);
        bad = __syncthreads_or(bad);
        met_odd = __syncthreads_or(met_odd);

        float gs = halves_sum(g);
        if (bad && (seq.cut || sees_bad_page(a, table, sp, begin, end, pos))) gs = __builtin_nanf("");
        const float inv = 1.0f / gs;
        const size_t o = (size_t)(seq.t0 + t) * a.Hq + q_head;
        if (row < rows) {
            if (plan.splits > 1 && hh == 0) part[(size_t)a.T * a.Hq * plan.splits * D + o * plan.splits + split] = gs;
            if (met_odd) {
#pragma unroll
                for (int d = 0; d < DT; ++d) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int ch = W::channel(d, i, hh), fr = wave * WR + c32;
                        if (flags[0][fr][ch / 32] >> (ch % 32) & 1) acc[d][i] += __builtin_inff();
                        if (flags[1][fr][ch / 32] >> (ch % 32) & 1) acc[d][i] -= __builtin_inff();
                    }
                }
            }
            // N neighbouring channels at a time
            constexpr int N = sizeof(T) == 2 || DT == 4 ? 4 : DT;
#pragma unroll
            for (int n = 0; n < 16 * DT / N; ++n) {
                float f[N];
                // bf16: a register quad of one accumulator; float32: a register of
                // every accumulator
                const int d0 = sizeof(T) == 2 ? n / 4 : 0, i0 = sizeof(T) == 2 ? n % 4 * 4 : n;
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] = sizeof(T) == 2 ? acc[d0][i0 + j] : acc[j][i0];
                const int ch = W::channel(d0, i0, hh);
                if (plan.splits > 1) {
                    put<N>(part + (o * plan.splits + split) * D + ch, f);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) f[j] = pos < 0 ? 0.f : f[j] * inv;   // pos < 0: sees no key
                    put<N>((T *)a.out + o * D + ch, f);
                }
            }
        }
        __syncthreads();   // the flags are read: another row tile may clear them
    }
}

template <typename T, int D> hipError_t launch(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    // Row tiles that share their keys stay on one XCD unless that leaves more
    // than an eighth of the XCDs' time empty, or several sequences, which may be
    // uneven, leave an XCD fewer than 8 of them.  bf16, D = 128: one sequence of
    // 8192 keys, 4096 rows of 32 heads to 4 1022 us on 4 XCDs, 570 in two pieces
    // each, 606 in eight; 16 sequences of up to 8192, 512 rows of 16 heads to 2
    // 394 whole, 307 in two pieces; 32 even ones of 4096, 256 rows of 32 heads to
    // 8 291 whole, 312 in two pieces.
    const long long units = (long long)a.S * a.Hkv * plan.splits;
    const auto more = [&](long long n) { return 7 * ((n + 7) / 8) > n || (a.S > 1 && n < 64); };
    int pieces = 1;
    while (pieces < 8 && 2 * pieces <= plan.tiles && more(units * pieces)) pieces *= 2;
    const long long blocks = (units * pieces + 7) / 8 * 8 * ((plan.tiles + pieces - 1) / pieces);
    if (!grid_fits(blocks, THREADS)) return hipErrorInvalidConfiguration;
    chunk_kernel<T, D><<<(unsigned)blocks, THREADS, 0, st>>>(a, plan, pieces, part);
    return hipGetLastError();
}

template <typename T> hipError_t launch_d(const PagedArgs &a, const PagedPlan &plan, int D, float *part, hipStream_t st)
{
    switch (D) {
    case 32: return launch<T, 32>(a, plan, part, st);
    case 64: return launch<T, 64>(a, plan, part, st);
    default: return launch<T, 128>(a, plan, part, st);
    }
}

}  // namespace

hipError_t paged_chunk(const PagedArgs &a, const PagedPlan &plan, int D, int is_bf16, float *part, hipStream_t st)
{
    return is_bf16 ? launch_d<bf16_t>(a, plan, D, part, st) : launch_d<float>(a, plan, D, part, st);
}

}  // namespace fm
