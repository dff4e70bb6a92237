// Fastmax attention of new tokens over a paged cache of standardised keys.
//
//     s_in = q^_i . k^_n,  w_in = f_p(tau s_in),
//     O_i = sum_n w_in v_n / sum_n w_in,
// n over the keys of the query's sequence that it sees: n <= pos_i, and with a
// window W and S first tokens, n > pos_i - W or n < S.  f_p needs no running
// maximum, so partial sums of a cut key range are simply added.
//
// Rows are the (token, query head) pairs that share a key head, 16 to an MFMA
// tile; a wave holds RT such tiles of q^ as B operands and walks over the
// keys, 32 at a time, straight from the cache into registers:
//   S^T = K Q^T    A: 16 keys (lane r16: key r16), accumulator: query r16,
//                  keys 4h .. 4h + 3 of the tile (lane = 16 h + r16)
//   O^T += V^T W^T B: exactly those accumulator lanes, two key tiles side by
//                  side (bf16) or one key of each row of lanes (float32)
// With channel r16 D/16 + j in row r16 of A for product j, a lane reads D/16
// neighbouring channels of the 8 keys whose weights it holds, and what MFMA
// wants transposed is transposed within the lane.  Nothing goes through LDS
// until the waves of a workgroup, which take key tiles in turn, add up.
//
// For single tokens HBM bounds it: every key and value is read once, whatever
// the number of heads that share it.  bf16, 32 heads to 8, D = 128: one sequence
// of 131072 keys 99 to 102 us (5.3 TB/s, join included), 61 of 4096 186 us
// (5.5), 61 of uneven lengths up to 8192 149 to 153 us (4.9: the last
// workgroups run alone); float32, 32 windows of 4096 keys, D = 64: 99 to 101 us (5.3).
// One sequence of 777 keys, 12 heads of 64: 8.3 us, one launch.  Chunks of prompts with many
// rows go to fm_paged_chunk.hip.
#include <hip/hip_runtime.h>

#include "fm_internal.h"
#include "fm_paged.h"
#include "fm_rows.h"
#include "fm_serve.h"

namespace fm {
namespace {

using namespace paged;

typedef short s4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;

template <typename T, int D> struct Mat;

// bf16: 16x16x32 MFMA (16x16x16 for the scores at D = 16).
template <int D> struct Mat<bf16_t, D> {
    static constexpr int QW = D >= 32 ? D / 32 : 1;
    static constexpr int VW = D / 16;                    // channels of a key per lane
    struct Q { u4 x[QW]; };
    struct K { u4 x[QW]; };
    struct V { uint32_t x[8][VW >= 2 ? VW / 2 : 1]; };   // [key of the lane][channel pair]

    static __device__ __forceinline__ void ld_row(const bf16_t *p, int h, u4 *x)
    {
        if constexpr (D >= 32) {
#pragma unroll
            for (int c = 0; c < QW; ++c) x[c] = *(const u4 *)(p + 32 * c + 8 * h);
        } else {
            const uint2 u = *(const uint2 *)(p + 4 * h);
            x[0] = u4{u.x, u.y, 0, 0};
        }
    }
    static __device__ __forceinline__ f4 scores(const K &k, const Q &q)
    {
        f4 s = {0.f, 0.f, 0.f, 0.f};
        if constexpr (D >= 32) {
#pragma unroll
            for (int c = 0; c < QW; ++c)
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, k.x[c]),
                                                            __builtin_bit_cast(b8, q.x[c]), s, 0, 0, 0);
        } else {
            const uint2 a = make_uint2(k.x[0][0], k.x[0][1]), b = make_uint2(q.x[0][0], q.x[0][1]);
            s = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s4, a), __builtin_bit_cast(s4, b),
                                                          s, 0, 0, 0);
        }
        return s;
    }
    // A lane's part of a score (added over the rows of lanes).
    static __device__ __forceinline__ float dot(const bf16_t *p, int h, const Q &q)
    {
        u4 k[QW];
        ld_row(p, h, k);
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < QW; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = k[c][i], b = q.x[c][i];
                s = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), s);
                s = fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), s);
            }
        return s;
    }
    // key i of the lane's eight: tile i / 4, key 4 h + i % 4
    static __device__ __forceinline__ void ld_v(const bf16_t *p, int r16, uint32_t *x)
    {
        p += r16 * VW;
        if constexpr (VW == 8) {
            const u4 u = *(const u4 *)p;
            x[0] = u[0]; x[1] = u[1]; x[2] = u[2]; x[3] = u[3];
        } else if constexpr (VW == 4) {
            const uint2 u = *(const uint2 *)p;
            x[0] = u.x; x[1] = u.y;
        } else if constexpr (VW == 2) {
            x[0] = *(const uint32_t *)p;
        } else {
            x[0] = *p;
        }
    }
    // Whether a value among the lane's is infinite or NaN: the largest
    // exponent, two channels at a time, sign shifted out.
    static constexpr bool PARTS = true;
    static __device__ __forceinline__ bool odd(const V &v)
    {
        typedef unsigned short us2 __attribute__((ext_vector_type(2)));
        us2 most = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (uint32_t x : v.x[i]) most = __builtin_elementwise_max(most, __builtin_bit_cast(us2, x) << 1);
        return most[0] >= 0xff00 || most[1] >= 0xff00;
    }
    // acc[j] += V^T W^T for channel r16 VW + j.  The weights enter as two
    // bf16 parts (16 bits of each): the second costs MFMA time that the
    // loads leave idle, and keeps the sums at float32's error.
    static __device__ __forceinline__ void add(f4 *acc, const V &v, const f4 *w)
    {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = w[i / 2][2 * (i % 2)], y = w[i / 2][2 * (i % 2) + 1];
            hi[i] = rows::pack2(x, y);
            lo[i] = rows::pack2(x - __uint_as_float(hi[i] << 16), y - __uint_as_float(hi[i] & 0xffff0000u));
        }
        const b8 bh = __builtin_bit_cast(b8, u4{hi[0], hi[1], hi[2], hi[3]});
        const b8 bl = __builtin_bit_cast(b8, u4{lo[0], lo[1], lo[2], lo[3]});
#pragma unroll
        for (int j = 0; j < VW; ++j) {
            // v_perm: bytes 0-3 of the second operand, 4-7 of the first
            const uint32_t sel = j % 2 ? 0x07060302u : 0x05040100u;
            u4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_perm(v.x[2 * i + 1][j / 2], v.x[2 * i][j / 2], sel);
            const b8 xa = __builtin_bit_cast(b8, x);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xa, bh, acc[j], 0, 0, 0);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xa, bl, acc[j], 0, 0, 0);
        }
    }
};

// float32: 16x16x4 MFMA, operands in full.
template <int D> struct Mat<float, D> {
    static constexpr int QW = D / 16;                    // 4-channel pieces of a lane's quarter row
    static constexpr int VW = D / 16;
    struct Q { f4 x[QW]; };
    struct K { f4 x[QW]; };
    struct V { float x[8][VW]; };

    // row of lanes h holds channels h D/4 .. (h + 1) D/4
    static __device__ __forceinline__ void ld_row(const float *p, int h, f4 *x)
    {
#pragma unroll
        for (int c = 0; c < QW; ++c) x[c] = *(const f4 *)(p + h * (D / 4) + 4 * c);
    }
    static __device__ __forceinline__ f4 scores(const K &k, const Q &q)
    {
        f4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < QW; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[c][i], q.x[c][i], s, 0, 0, 0);
        return s;
    }
    static __device__ __forceinline__ float dot(const float *p, int h, const Q &q)
    {
        f4 k[QW];
        ld_row(p, h, k);
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < QW; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) s = fmaf(k[c][i], q.x[c][i], s);
        return s;
    }
    static __device__ __forceinline__ void ld_v(const float *p, int r16, float *x)
    {
        p += r16 * VW;
        if constexpr (VW >= 4) {
#pragma unroll
            for (int j = 0; j < VW; j += 4) {
                const f4 u = *(const f4 *)(p + j);
                x[j] = u[0]; x[j + 1] = u[1]; x[j + 2] = u[2]; x[j + 3] = u[3];
            }
        } else if constexpr (VW == 2) {
            const float2 u = *(const float2 *)p;
            x[0] = u.x; x[1] = u.y;
        } else {
            x[0] = *p;
        }
    }
    static constexpr bool PARTS = false;
    static __device__ __forceinline__ bool odd(const V &v)
    {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (float x : v.x[i]) most = max(most, __float_as_uint(x) << 1);
        return most >= 0xff000000u;
    }
    static __device__ __forceinline__ void add(f4 *acc, const V &v, const f4 *w)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < VW; ++j)
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.x[i][j], w[i / 4][i % 4], acc[j], 0, 0, 0);
    }
};

// MULTI: rows of several tokens may share a tile, so a key can be visible to
// some rows of a tile and not to others.
// At D = 128 registers are bounded for as many waves as pay on a SIMD: three in
// bf16, two in float32 (61 sequences of up to 8192 keys, 8 heads, float32 309 us;
// one 367).
template <typename T, int D, int RT, bool MULTI, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D == 128 && RT == 1 && WAVES == 4 ? (sizeof(T) == 2 ? 3 : 2) : 1)
void paged_kernel(PagedArgs a, PagedPlan plan, float *part)
{
    using M = Mat<T, D>;
    constexpr int VW = M::VW, ROWS = 16 * RT, RS = D + 4;
    __shared__ float red[WAVES][16][RS];
    __shared__ float gred[WAVES][16];

    // Splits last: later ones are empty in shorter sequences, and workgroups are
    // dealt out to the XCDs in turn.
    int id = blockIdx.x;
    const int head = id % a.Hkv;
    id /= a.Hkv;
    const int s = id % a.S;
    id /= a.S;
    const int tile0 = id % plan.tiles, split = id / plan.tiles;
    const int wave = scalar(threadIdx.x / 64), lane = threadIdx.x % 64, h = lane / 16, r16 = lane % 16;
    const Seq seq = seq_of(a, s);
    const int rows = seq.count * a.group, page_mask = (1 << a.page_shift) - 1;
    const T *kc = (const T *)a.k + head * a.cache.head, *vc = (const T *)a.v + head * a.cache.head;
    const int32_t *table = a.table + (size_t)s * a.table_cols;
    const int token = (int)a.cache.token;

    // max_q sets the grid; a sequence with more new tokens goes round again
    for (int r0 = tile0 * ROWS; r0 < rows; r0 += plan.tiles * ROWS) {
        const Span sp = scalar(span_of_rows(a, seq, r0, ROWS));
        const int begin = split * plan.chunk;
        const int end = split == plan.splits - 1 ? sp.tiles : min(sp.tiles, begin + plan.chunk);
        if (begin >= sp.tiles && split > 0) continue;   // the join knows

        typename M::Q q[RT];
        int pos[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = min(r0 + 16 * r + r16, rows - 1);
            const int t = row / a.group;
            pos[r] = seq.len - seq.count + t;
            M::ld_row((const T *)a.q + (seq.t0 + t) * a.q_token + (head * a.group + row - t * a.group) * a.q_head,
                      h, q[r].x);
        }
        f4 acc[RT][VW];
        float g[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            g[r] = 0.f;
#pragma unroll
            for (int j = 0; j < VW; ++j) acc[r][j] = f4{0.f, 0.f, 0.f, 0.f};
        }
        const int first = scalar(seq.len - seq.count + r0 / a.group), last = sp.end - 1;
        // Key tiles [whole, whole_end) exist in full and every row sees all their
        // keys; elsewhere keys are clamped and weights masked.
        const int shift = sp.low - sp.sink_tiles;   // from a tile's number here to its own
        const int whole = a.window < sp.end ? max(sp.sink_tiles, (last - a.window) / KT + 1 - shift) : 0;
        const int whole_end = min(end, (first + 1) / KT - shift);
        bool bad = seq.cut;

        // The wave's steps of two key tiles, 32 steps at a time: where they begin
        // in the cache, a tile to a lane, so that no step waits for the page
        // table.
        for (int b0 = begin + 2 * wave; b0 < end; b0 += 64 * WAVES) {
            const int mine = sp.tile(min(b0 + lane / 2 * (2 * WAVES) + lane % 2, end - 1)) * KT;
            int page = table[mine >> a.page_shift];
            if ((unsigned)page >= (unsigned)a.pages) {
                bad = true;
                page = 0;
            }
            const long long at = page * a.cache.batch + (mine & page_mask) * a.cache.token;
            for (int n = 0; n < 32; ++n) {
                const int i0 = b0 + n * (2 * WAVES);
                if (i0 >= end) break;
                typename M::K k[2];
                typename M::V v;
                const bool all = i0 >= whole && i0 + 2 <= whole_end;
                int base[2];   // of the key tiles; past every position if there is none
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const long long from =
                        (long long)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(at >> 32), 2 * n + i) << 32 |
                                    (uint32_t)__builtin_amdgcn_readlane((int)at, 2 * n + i));
                    const T *kp = kc + from, *vp = vc + from;
                    const int n0 = sp.tile(min(i0 + i, end - 1)) * KT;
                    base[i] = i0 + i < end ? n0 : INT32_MAX - KT;
                    int kr = r16, vr[4] = {4 * h, 4 * h + 1, 4 * h + 2, 4 * h + 3};
                    if (!all) {
                        kr = sp.read(n0 + kr, n0 + KT - 1) - n0;
#pragma unroll
                        for (int j = 0; j < 4; ++j) vr[j] = sp.read(n0 + vr[j], n0 + KT - 1) - n0;
                    }
                    M::ld_row(kp + kr * token, h, k[i].x);
#pragma unroll
                    for (int j = 0; j < 4; ++j) M::ld_v(vp + vr[j] * token, r16, v.x[4 * i + j]);
                }
                // A value that is infinite or NaN takes the step out of MFMA: a row
                // whose weight is 0 because it does not see the key would get NaN,
                // and so would infinity times a weight's second part.  Without
                // either (float32, one token: its rows see the same keys) what was
                // read in place of a key that is not seen becomes 0, as its weight.
                if constexpr (!M::PARTS && !MULTI) {
                    if (!all) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (visible(base[i / 4] + 4 * h + i % 4, pos[0], a.window, a.sinks)) continue;
#pragma unroll
                            for (auto &x : v.x[i]) x = 0.f;
                        }
                    }
                }
                const bool odd = (M::PARTS || (MULTI && !all)) && __any(M::odd(v));
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    f4 w[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const f4 x = M::scores(k[i], q[r]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            w[i][j] = fmaf(fmaf(x[j], a.c2, a.c1), x[j], 1.0f);
                            if (!all && !visible(base[i] + 4 * h + j, pos[r], a.window, a.sinks)) w[i][j] = 0.f;
                            g[r] += w[i][j];
                        }
                    }
                    if (!odd) {
                        M::add(acc[r], v, w);
                        continue;
                    }
                    // each row adds the keys it sees, one by one
#pragma unroll 1
                    for (int i = 0; i < 2 * KT; ++i) {
                        const int key = (i < KT ? base[0] : base[1]) + i % KT;
                        if (key >= sp.end) continue;
                        const int pg = table[key >> a.page_shift];
                        if ((unsigned)pg >= (unsigned)a.pages) continue;
                        const long long from = pg * a.cache.batch + (key & page_mask) * a.cache.token;
                        const float x = rows4_sum(M::dot(kc + from, h, q[r]));
                        if (!visible(key, pos[r], a.window, a.sinks)) continue;
                        const float wk = fmaf(fmaf(x, a.c2, a.c1), x, 1.0f);
                        const T *vp = vc + from + h * (D / 4);
#pragma unroll
                        for (int d = 0; d < D / 4; ++d)
                            acc[r][d % VW][d / VW] = fmaf(wk, io<T>::ld(vp, d), acc[r][d % VW][d / VW]);
                    }
                }
            }
        }
        bad = __any(bad);

        // the waves' sums, one row tile at a time
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float gs = rows4_sum(g[r]);
            if (bad && (seq.cut || sees_bad_page(a, table, sp, begin, end, pos[r]))) gs = __builtin_nanf("");
            __syncthreads();
            if (h == 0) gred[wave][r16] = gs;
#pragma unroll
            for (int d = 0; d < D / 4; ++d) red[wave][r16][h * (D / 4) + d] = acc[r][d % VW][d / VW];
            __syncthreads();
            const int rr = threadIdx.x / 16, c = threadIdx.x % 16 * VW, row = r0 + 16 * r + rr;
            if (rr < 16 && row < rows) {
                float f[VW], gg = 0.f;
#pragma unroll
                for (int j = 0; j < VW; ++j) f[j] = 0.f;
#pragma unroll
                for (int v = 0; v < WAVES; ++v) {
                    gg += gred[v][rr];
#pragma unroll
                    for (int j = 0; j < VW; ++j) f[j] += red[v][rr][c + j];
                }
                const int t = row / a.group;
                const size_t o = (size_t)(seq.t0 + t) * a.Hq + head * a.group + row - t * a.group;
                if (plan.splits == 1) {
                    const bool none = seq.len - seq.count + t < 0;   // sees no key
                    T *out = (T *)a.out + o * D + c;
#pragma unroll
                    for (int j = 0; j < VW; ++j) io<T>::st(out, j, none ? 0.f : f[j] / gg);
                } else {
                    float *p = part + (o * plan.splits + split) * D + c;
#pragma unroll
                    for (int j = 0; j < VW; ++j) p[j] = f[j];
                    if (c == 0) part[(size_t)a.T * a.Hq * plan.splits * D + o * plan.splits + split] = gg;
                }
            }
        }
    }
}

// Adds the splits' sums: a row to RW waves, 16 lanes side by side over its
// channels and 4 RW of these over its splits, four splits in flight in each.
// Latency bounds it: 32 rows of 128 splits 14 us with one wave each, 7 with
// four; 1952 rows of 8 splits 9 us with one.
template <typename T, int D, int RW>
__global__ __launch_bounds__(THREADS) void join_kernel(PagedArgs a, PagedPlan plan, const float *part)
{
    constexpr int VW = D / 16, U = 4, L = 4 * RW, ROWS = WAVES / RW;
    __shared__ float red[WAVES][D + 1];
    const int s = blockIdx.y;
    const Seq seq = seq_of(a, s);
    const long long n = (long long)seq.count * a.Hq;
    const int wave = threadIdx.x / 64, c = threadIdx.x % 16 * VW, l = threadIdx.x / 16 % L;
    const float *gpart = part + (size_t)a.T * a.Hq * plan.splits * D;
    for (long long i0 = (long long)blockIdx.x * ROWS; i0 < n; i0 += (long long)gridDim.x * ROWS) {
        const long long i = min(i0 + wave / RW, n - 1);
        const int t = (int)(i / a.Hq), head = (int)(i - (long long)t * a.Hq);
        const int row = t * a.group + head % a.group;
        const Span sp = span_of_rows(a, seq, row / plan.rows * plan.rows, plan.rows);
        const int used = max(1, min(plan.splits, (sp.tiles + plan.chunk - 1) / plan.chunk));
        const size_t o = (size_t)(seq.t0 + t) * a.Hq + head;
        const float *p = part + o * plan.splits * D + c, *gp = gpart + o * plan.splits;
        float f[VW], g = 0.f;
#pragma unroll
        for (int j = 0; j < VW; ++j) f[j] = 0.f;
        for (int k = l; k < used; k += L * U) {
            float x[U][VW], y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = min(k + L * u, used - 1);
                y[u] = gp[at];
#pragma unroll
                for (int j = 0; j < VW; ++j) x[u][j] = p[(size_t)at * D + j];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k + L * u >= used) break;
                g += y[u];
#pragma unroll
                for (int j = 0; j < VW; ++j) f[j] += x[u][j];
            }
        }
        g = rows4_sum(g);
#pragma unroll
        for (int j = 0; j < VW; ++j) f[j] = rows4_sum(f[j]);
        if constexpr (RW > 1) {
            __syncthreads();
            if (l % 4 == 0) {
                red[wave][D] = g;
#pragma unroll
                for (int j = 0; j < VW; ++j) red[wave][c + j] = f[j];
            }
            __syncthreads();
            if (l == 0) {
#pragma unroll
                for (int w = 1; w < RW; ++w) {
                    g += red[wave + w][D];
#pragma unroll
                    for (int j = 0; j < VW; ++j) f[j] += red[wave + w][c + j];
                }
            }
        }
        if (l || i0 + wave / RW >= n) continue;
        const bool none = seq.len - seq.count + t < 0;
        T *out = (T *)a.out + o * D + c;
#pragma unroll
        for (int j = 0; j < VW; ++j) io<T>::st(out, j, none ? 0.f : f[j] / g);
    }
}

template <typename T, int D, int RT, int W = WAVES>
hipError_t launch_rt(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    const long long blocks = (long long)plan.splits * plan.tiles * a.Hkv * a.S;
    if (!grid_fits(blocks, 64 * W)) return hipErrorInvalidConfiguration;
    if (a.q_start) paged_kernel<T, D, RT, true, W><<<(unsigned)blocks, 64 * W, 0, st>>>(a, plan, part);
    else paged_kernel<T, D, RT, false, W><<<(unsigned)blocks, 64 * W, 0, st>>>(a, plan, part);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    hipError_t e;
    if (plan.chunk_kernel) e = paged_chunk(a, plan, D, sizeof(T) == 2, part, st);
    else if (plan.waves == 8) e = launch_rt<T, D, 1, 8>(a, plan, part, st);
    else if (plan.rows == 16) e = launch_rt<T, D, 1>(a, plan, part, st);
    else if (plan.rows == 32) e = launch_rt<T, D, 2>(a, plan, part, st);
    else if constexpr (sizeof(T) * D <= 256) e = launch_rt<T, D, 4>(a, plan, part, st);
    else e = hipErrorInvalidValue;   // no plan has such rows
    if (e != hipSuccess || plan.splits == 1) return e;
    // a workgroup to a row where there are more splits than a wave has in flight
    const int per = plan.splits > 16 ? 1 : WAVES;
    const long long rows = (long long)plan.rows * plan.tiles / a.group * a.Hq;
    const long long most = (long long)a.T * a.Hq;   // of one sequence
    const dim3 grid((unsigned)(((rows < most ? rows : most) + per - 1) / per), (unsigned)a.S);
    if (per == 1) join_kernel<T, D, WAVES><<<grid, THREADS, 0, st>>>(a, plan, part);
    else join_kernel<T, D, 1><<<grid, THREADS, 0, st>>>(a, plan, part);
    return hipGetLastError();
}

template <typename T> hipError_t launch_d(const PagedArgs &a, const PagedPlan &plan, int D, float *part, hipStream_t st)
{
    switch (D) {
    case 16: return launch<T, 16>(a, plan, part, st);
    case 32: return launch<T, 32>(a, plan, part, st);
    case 64: return launch<T, 64>(a, plan, part, st);
    default: return launch<T, 128>(a, plan, part, st);
    }
}

}  // namespace

PagedPlan paged_plan(int S, int Hq, int Hkv, int D, int is_bf16, int max_q, int max_len, int window,
                     int sinks)
{
    PagedPlan plan;
    const long long rows = (long long)max_q * (Hq / Hkv);
    // The chunk kernel against this one, 8 sequences of 4096 keys, 8 key heads:
    // 32 rows (8 tokens, 4 query heads to a key head) bf16 D = 128 43 against
    // 36 us, D = 64 29 against 20, D = 32 23 against 15; 48 to 64 rows bf16
    // D = 128 44 against 51, D = 64 31 against 36, D = 32 24 against 21, float32
    // D = 128 154 against 129, D = 64 84 against 61; 128 rows D = 128 49 against
    // 50 and more beyond.  Single tokens stay here whatever their heads.
    plan.chunk_kernel = D >= 32 && max_q > 1 && (rows > 64 || (rows > 32 && is_bf16 && D >= 64));
    plan.rows = plan.chunk_kernel ? CHUNK_ROWS : rows <= 16 ? 16 : rows <= 32 || (!is_bf16 && D == 128) ? 32 : 64;
    plan.waves = WAVES;
    // max_q holds for the longest sequence and may be all of T, so most row tiles
    // of a grid may be empty: past 2^18 workgroups it has no more of them, and
    // the rows behind them are taken in rounds.  (An empty workgroup costs a ns:
    // 1024 prompts of 128 tokens, 8 key heads, D = 32, max_q left out 594 us, 1367
    // with up to 2^20, 8910 with 2^23; 359 with the max_q that they have.  One
    // prompt of 8192 tokens among 1023 of up to 40, D = 64: 810, 1701, 2811 us,
    // and 2530 with up to 2^16.)
    const long long pairs = (long long)S * Hkv, most = (1 << 18) / pairs > 1 ? (1 << 18) / pairs : 1;
    const long long all = (rows + plan.rows - 1) / plan.rows, tiles = all < most ? all : most;
    // the most key tiles that a row tile can see
    const long long tokens = (long long)plan.rows * Hkv / Hq + 2;
    const long long seen = (long long)window + tokens + 2 * KT + sinks;
    const long long keys = max_len < seen ? max_len : seen;
    const long long key_tiles = (keys + KT - 1) / KT;
    // Splits, where (sequence, head, row tile) leave CUs idle: toward 2048
    // workgroups (1024 of the chunk kernel's, which are two to a CU) while
    // 1024 keys (float32: 512) are left for each, toward 512 below that, down
    // to 256 keys.  Less costs more in partial sums than the CUs gain: one
    // sequence of 131072 keys, 8 heads, D = 128: 112 us in 1024 workgroups,
    // 127 in 2048; 4 of 16384: 29 us in 512, 39 in 2048; 61 of up to 8192:
    // 155 us in up to 2440, 171 in 1464.
    const long long base = tiles * pairs;
    const auto toward = [&](long long target, long long least) {
        const long long by_target = (target + base - 1) / base, by_size = (key_tiles + least - 1) / least;
        return by_target < by_size ? by_target : by_size;
    };
    long long splits = 1;
    if (plan.chunk_kernel) {
        splits = toward(1024, 64);
        for (const int t : {512, 256}) {
            const long long few = toward(t, t / 16);
            if (splits * base < t && splits < few) splits = few;
        }
    } else if (base < 1024) {
        // Eight waves and one launch where a second one costs more than it
        // gives: up to a workgroup per CU while keys and values of a head are
        // at most 256 KB, beyond that while twice the least above is not
        // passed and the workgroups' registers fit the CUs.  bf16: one
        // sequence of 512 keys, 12 heads of 64 7.0 us, 7.9 in two splits (and
        // 12 against 17 a call); of 1024 keys, 8 heads of 128 13 against 9, so
        // split; 32 of 512 keys 15 against 19; 64 of up to 512, 4 heads of 64
        // 7.7 against 11; but 100 of up to 512, 8 heads of 128 26 against 18
        // (four waves).  Rows of at most 128 bytes (registers for more waves)
        // take eight waves up to 1023 workgroups, against four and splits: bf16,
        // 125 of 2048 keys, 8 heads of 64 95 against 105 (uneven: 43 against 51), of
        // 1024 50 against 53 (26 against 24); 75 to 120 of 2048, heads of 32 36 against
        // 40 (22 against 31), of 16 30 against 37; float32 heads of 32, 1024 keys 37
        // against 41 (23 against 33); at 300 keys 12.5 against 11.4, 9.2 against 7.8
        // and 9.8 against 8.5.  Under 256 keys four waves do: 60 keys 4.8, eight 5.4.
        const long long least = is_bf16 ? 64 : 32, row = (is_bf16 ? 2 : 4) * D;
        const bool one = base < 256 ? key_tiles * KT * row <= 128 << 10
                                    : key_tiles <= 2 * least && (base <= 512 || row <= 128);
        if (plan.rows == 16 && key_tiles > 16 && one) {
            plan.waves = 8;
        } else {
            splits = toward(2048, least);
            const long long few = toward(512, 16);
            if (splits * base < 512 && splits < few) splits = few;
        }
    }
    if (splits < 1) splits = 1;
    long long chunk = (key_tiles + splits - 1) / splits;
    chunk = (chunk + 2 * plan.waves - 1) / (2 * plan.waves) * (2 * plan.waves);
    plan.tiles = (int)tiles;
    plan.chunk = (int)chunk;
    plan.splits = (int)((key_tiles + chunk - 1) / chunk);
    return plan;
}

size_t paged_workspace(const PagedPlan &plan, int T, int Hq, int D)
{
    return plan.splits == 1 ? 0 : (size_t)T * Hq * plan.splits * (D + 1) * sizeof(float);
}

hipError_t paged_fwd(const PagedArgs &a, const PagedPlan &plan, int D, int is_bf16, void *ws, hipStream_t st)
{
    return is_bf16 ? launch_d<bf16_t>(a, plan, D, (float *)ws, st) : launch_d<float>(a, plan, D, (float *)ws, st);
}

}  // namespace fm
