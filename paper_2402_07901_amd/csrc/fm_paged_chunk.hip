// Paged attention of many rows of a sequence (chunks of prompts), bf16.
//
// MFMA bounds it, so keys and values are staged in LDS for a workgroup's 128
// rows, 64 keys at a time, and each of its four waves works on 32 rows with
// 32x32x16 tiles:
//   S^T = K Q^T    A: 32 keys (one 16-byte LDS read per lane and 16 channels),
//                  B: q^ of 32 rows, in registers throughout
//   O^T += V^T W^T B: the weights, which the accumulator layout of S^T holds
//                  where B wants them if a 16-key step takes keys
//                  {4h..4h+3, 8+4h..8+4h+3} for the lanes of half h; A: the
//                  same keys of 32 channels, through the transposing LDS read
// (lane = 32 h + c32; accumulator register i: column c32, row 8 (i/4) + 4 h + i%4).
// The next 64 keys go straight to the other LDS buffer (global_load_lds) while
// these are worked on.  Registers: two waves on a SIMD, from two workgroups,
// whose products and weights overlap.  64 rows per wave read LDS half as often
// but leave one wave on a SIMD at D = 128: 904 against 1003 TFLOP/s.
//
// LDS rows are D channels with no padding; the 16-byte piece c of row r lies
// at piece c ^ swizzle(r), which puts 8 consecutive rows' piece c (score
// operands) and pieces c, c + 1 of 4 consecutive rows (value operands) on
// distinct banks.
//
// The weights enter as bf16, and the row's sum adds the rounded ones: what is
// rounded is the weights of an average, whose errors of 2^-9 each largely
// cancel, below the rounding of the output itself; two parts, as in the
// register kernel, would add half the MFMA work.
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
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef unsigned short us2 __attribute__((ext_vector_type(2)));

constexpr int THREADS = 256;
constexpr int KB = 64;   // keys per LDS buffer
constexpr int WAIT_LOADS = 0x0f70;   // vmcnt(0), the other counters at their most

template <int D> __device__ __forceinline__ int swizzle(int r)
{
    if constexpr (D >= 64) return (r & 3) << 1 | (r >> 2 & 1);
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

template <int D>
__global__ __launch_bounds__(THREADS, 2) void chunk_kernel(PagedArgs a, PagedPlan plan, float *part)
{
    constexpr int ROWS = CHUNK_ROWS, WR = ROWS / 4;   // rows of a workgroup, of a wave
    constexpr int C = D / 8;                       // 16-byte pieces of a row
    constexpr int KC = D / 16, DT = D / 32;
    constexpr int LR = 64 / C;                     // rows that a wave's load covers
    constexpr int LN = KB / LR / 4;                // loads of a wave, of keys and of values
    // two buffers
    __shared__ u4 keys0[KB * C], keys1[KB * C], values0[KB * C], values1[KB * C];
    // channels of a row that met +infinity, -infinity (both: NaN) where not
    // every row sees the key
    __shared__ uint32_t flags[2][ROWS][DT];

    // Workgroups of one (sequence, key head) read the same keys: they go to the
    // same XCD (workgroups are dealt out to the 8 XCDs in turn).  Late row
    // tiles see the most keys and start first.
    int id = blockIdx.x / 8;
    const int row_tile = plan.tiles - 1 - id % plan.tiles;
    id /= plan.tiles;
    const int split = id % plan.splits;
    const int pair = id / plan.splits * 8 + blockIdx.x % 8;
    if (pair >= a.S * a.Hkv) return;
    const int head = pair % a.Hkv, s = pair / a.Hkv;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = threadIdx.x % 64, hh = lane / 32, c32 = lane % 32;
    const Seq seq = seq_of(a, s);
    const int rows = seq.count * a.group, page_mask = (1 << a.page_shift) - 1;
    const bf16_t *kc = (const bf16_t *)a.k + head * a.cache.head, *vc = (const bf16_t *)a.v + head * a.cache.head;
    const int32_t *table = a.table + (size_t)s * a.table_cols;

    uint32_t lane_at[LN];   // bytes from a tile's first row to what the lane loads
#pragma unroll
    for (int i = 0; i < LN; ++i) {
        const int r = (wave + 4 * i) * LR + lane / C;
        lane_at[i] = 2 * (r % KT * (int)a.cache.token + 8 * (lane % C ^ swizzle<D>(r)));
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
        u4 q[KC];
        f16v acc[DT];
        float g = 0.f;
        {
            const bf16_t *p = (const bf16_t *)a.q + (seq.t0 + t) * a.q_token + q_head * a.q_head + 8 * hh;
#pragma unroll
            for (int k = 0; k < KC; ++k) q[k] = *(const u4 *)(p + 16 * k);
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] = f16v{};
        }
        bool bad = seq.cut;
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
                    off = 2 * ((sp.read(n0 + r % KT, n0 + KT - 1) - n0) * (int)a.cache.token + 8 * (lane % C ^ swizzle<D>(r)));
                }
                to_lds((const char *)(kc + from) + off, kd + l0 * C);
                to_lds((const char *)(vc + from) + off, vd + l0 * C);
            }
        };
        const auto unseen = [&](int i0) { return i0 < whole || i0 + KB / KT > whole_end; };
        // An infinity or a NaN among values that some row may not see: weight 0
        // would make it NaN there, so it leaves the buffer, and the rows that
        // do see it are marked.
        const auto screen = [&](int i0, u4 *vd) {
#pragma unroll 1
            for (int piece = threadIdx.x; piece < KB * C; piece += THREADS) {
                const u4 y = vd[piece];
                us2 most = {0, 0};   // largest exponent, sign shifted out
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(us2, (uint32_t)y[j]) << 1);
                if (most[0] < 0xff00 && most[1] < 0xff00) continue;
                const int r = piece / C, c = piece % C ^ swizzle<D>(r);
                bf16_t *x = (bf16_t *)&vd[piece];
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {
                    const bf16_t v = x[e];
                    if ((v & 0x7f80) != 0x7f80) continue;
                    x[e] = 0;
                    if (i0 + r / KT >= end) continue;
                    const int n = sp.tile(i0 + r / KT) * KT + r % KT;
#pragma unroll 1
                    for (int i = 0; i < ROWS && r0 + i < rows; ++i) {
                        const int t = (r0 + i) / a.group;
                        if (!visible(n, pos0 + t, a.window, a.sinks)) continue;
                        const bool nan = (v & 0x7f) != 0;
                        bool neg = v >> 15;
                        if (!nan && a.c2 == 0.f) {   // first order: the weight has a sign
                            const bf16_t *qp = (const bf16_t *)a.q + (seq.t0 + t) * a.q_token +
                                               (head * a.group + r0 + i - t * a.group) * a.q_head;
                            const int page = min((unsigned)table[n >> a.page_shift], (unsigned)a.pages - 1);
                            const bf16_t *kp = kc + page * a.cache.batch + (n & page_mask) * a.cache.token;
                            float dot = 0.f;
#pragma unroll 1
                            for (int d = 0; d < D; ++d) dot = fmaf(bf16_to_f32(qp[d]), bf16_to_f32(kp[d]), dot);
                            neg ^= fmaf(dot, a.c1, 1.0f) < 0.f;
                        }
                        const int ch = 8 * c + e;
                        if (nan || !neg) atomicOr(&flags[0][i][ch / 32], 1u << (ch % 32));
                        if (nan || neg) atomicOr(&flags[1][i][ch / 32], 1u << (ch % 32));
                    }
                }
            }
            __syncthreads();
        };

        // Operands from LDS: 32 keys kb for the scores, and under the weights.
        const auto keys_of = [&](const u4 *kl, int kb, u4 *k) {
#pragma unroll
            for (int i = 0; i < KC; ++i)
                k[i] = kl[(32 * kb + c32) * C + ((2 * i + hh) ^ swizzle<D>(c32))];
        };
        const auto values_of = [&](const u4 *vb, int kb, u4 (&v)[2][DT]) {
            const s4 *vl = (const s4 *)vb;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    typedef s4 __attribute__((address_space(3))) *lp;
                    const int j = lane >> 2 & 3, r = 32 * kb + 16 * m + 4 * hh + j;
                    const int c = 4 * d + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
                    const int at = 2 * (r * C + (c ^ swizzle<D>(4 * hh + j))) + (lane & 1);
                    const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(vl + at));
                    const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(vl + at + 2 * 8 * C));
                    const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
                    v[m][d] = u4{l.x, l.y, h.x, h.y};
                }
            }
        };
        const auto score = [&](const u4 *k) {
            f16v x = f16v{};
#pragma unroll
            for (int i = 0; i < KC; ++i) x = mma(k[i], q[i], x);
            return x;
        };
        // Weights from scores, rounded, and summed so.
        const auto weigh = [&](const f16v &x, u4 (&w)[2], auto &&seen) {
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float y[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float z = x[i + j];
                    y[j] = seen(i + j) ? fmaf(fmaf(z, a.c2, a.c1), z, 1.0f) : 0.f;
                }
                const uint32_t u = rows::pack2(y[0], y[1]);
                w[i / 8][i / 2 % 4] = u;
                const b2 one = {(__bf16)1.0f, (__bf16)1.0f};
                g = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, u), one, g, false);
            }
        };
        const auto add = [&](const u4 (&v)[2][DT], const u4 (&w)[2]) {
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[d] = mma(v[m][d], w[m], acc[d]);
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
                    u4 ka[KC], va[2][DT], w[2];
                    keys_of(k, kb, ka);
                    const f16v x = score(ka);
                    values_of(v, kb, va);
                    if (all) {
                        weigh(x, w, [](int) { return true; });
                    } else {
                        int base[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int it = i0 + 2 * kb + i;
                            base[i] = it < end ? sp.tile(it) * KT : INT32_MAX - KT;   // past every position
                        }
                        weigh(x, w, [&](int i) {
                            return visible(base[i / 8] + 8 * (i / 4 % 2) + 4 * hh + i % 4, pos, a.window, a.sinks);
                        });
                    }
                    add(va, w);
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

        float gs = halves_sum(g);
        if (bad) gs = __builtin_nanf("");
        const float inv = 1.0f / gs;
        const size_t o = (size_t)(seq.t0 + t) * a.Hq + q_head;
        if (row < rows) {
            if (plan.splits > 1 && hh == 0) part[(size_t)a.T * a.Hq * plan.splits * D + o * plan.splits + split] = gs;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                f16v f = acc[d];
                const uint32_t plus = flags[0][wave * WR + c32][d], minus = flags[1][wave * WR + c32][d];
                if (plus | minus) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int bit = 8 * (i / 4) + 4 * hh + i % 4;
                        if (plus >> bit & 1) f[i] += __builtin_inff();
                        if (minus >> bit & 1) f[i] -= __builtin_inff();
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int ch = 32 * d + 8 * e + 4 * hh;
                    if (plan.splits > 1) {
                        *(float4 *)(part + (o * plan.splits + split) * D + ch) =
                            make_float4(f[4 * e], f[4 * e + 1], f[4 * e + 2], f[4 * e + 3]);
                    } else {
                        const uint32_t lo = rows::pack2(f[4 * e] * inv, f[4 * e + 1] * inv);
                        const uint32_t hi = rows::pack2(f[4 * e + 2] * inv, f[4 * e + 3] * inv);
                        // a row before the sequence sees no key
                        *(uint2 *)((bf16_t *)a.out + o * D + ch) = pos < 0 ? make_uint2(0, 0) : make_uint2(lo, hi);
                    }
                }
            }
        }
        __syncthreads();   // the flags are read: another row tile may clear them
    }
}

template <int D> hipError_t launch(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    const long long pairs = ((long long)a.S * a.Hkv + 7) / 8 * 8;
    const long long blocks = pairs * plan.tiles * plan.splits;
    if (!grid_fits(blocks, THREADS)) return hipErrorInvalidConfiguration;
    chunk_kernel<D><<<(unsigned)blocks, THREADS, 0, st>>>(a, plan, part);
    return hipGetLastError();
}

}  // namespace

hipError_t paged_chunk(const PagedArgs &a, const PagedPlan &plan, int D, float *part, hipStream_t st)
{
    switch (D) {
    case 32: return launch<32>(a, plan, part, st);
    case 64: return launch<64>(a, plan, part, st);
    default: return launch<128>(a, plan, part, st);
    }
}

}  // namespace fm
