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
// Every key that is loaded is one that some row of the tile sees: lanes whose
// key is past the end, or in the gap behind the window, read such a key
// instead and get weight 0, so what lies in unused or evicted slots never
// enters a product.
#include <hip/hip_runtime.h>

#include "fm_internal.h"
#include "fm_rows.h"
#include "fm_serve.h"

namespace fm {
namespace {

typedef short s4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int KT = 16;   // keys per tile

// The key tiles that a range of query positions [first, last] reads, in
// order: `sink_tiles` from the start of the sequence, then from tile `low` on.
struct Span {
    int end;          // keys before this one exist for some row
    int low_key;      // window: the lowest key the first position sees (0: no gap)
    int sinks;        // first tokens that stay visible
    int sink_tiles, low, tiles;
    __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : i - sink_tiles + low; }
    // The key to read in place of key n of the tile that ends at `last`: n
    // itself unless no row sees it.
    __device__ __forceinline__ int read(int n, int last) const
    {
        if (n >= sinks && n < low_key) n = low_key <= last ? low_key : sinks - 1;
        return min(n, end - 1);
    }
};

__device__ __forceinline__ Span span_of(int first, int last, int window, int sinks)
{
    Span s;
    s.end = last + 1;
    s.sinks = min(sinks, s.end);
    s.low_key = max(0, first - window + 1);
    if (s.low_key <= s.sinks) s.low_key = 0;
    s.low = s.low_key / KT;
    s.sink_tiles = s.low_key ? (s.sinks + KT - 1) / KT : 0;
    if (s.sink_tiles >= s.low) s.sink_tiles = s.low = 0;
    s.tiles = last < 0 ? 0 : s.sink_tiles + (s.end + KT - 1) / KT - s.low;
    return s;
}

__device__ __forceinline__ bool visible(int n, int pos, int window, int sinks)
{
    return n <= pos && (n > pos - window || n < sinks);
}

// A sequence's new tokens: rows [t0, t0 + count) of q, the last at len - 1.
struct Seq {
    int t0, count, len;
    bool cut;   // longer than its row of the page table
};

__device__ __forceinline__ Seq seq_of(const PagedArgs &a, int s)
{
    Seq q;
    q.t0 = a.q_start ? min(max(a.q_start[s], 0), a.T) : s;
    q.count = a.q_start ? min(max(a.q_start[s + 1], q.t0), a.T) - q.t0 : 1;
    const long long room = (long long)a.table_cols << a.page_shift;
    q.len = max(a.lens[s], 0);
    q.cut = q.len > room;
    q.len = (int)min((long long)q.len, room);
    return q;
}

// Positions of the row tile [r0, r0 + 16 RT) of a sequence.
__device__ __forceinline__ Span span_of_rows(const PagedArgs &a, const Seq &q, int r0, int rows)
{
    const int first = q.len - q.count + r0 / a.group;
    const int last = q.len - q.count + min(q.count - 1, (r0 + rows - 1) / a.group);
    return span_of(first, last, a.window, a.sinks);
}

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
template <typename T, int D, int RT, bool MULTI>
__global__ __launch_bounds__(THREADS) void paged_kernel(PagedArgs a, PagedPlan plan, float *part)
{
    using M = Mat<T, D>;
    constexpr int VW = M::VW, ROWS = 16 * RT, RS = D + 4;
    __shared__ float red[WAVES][16][RS];
    __shared__ float gred[WAVES][16];

    int id = blockIdx.x;
    const int split = id % plan.splits;
    id /= plan.splits;
    const int tile0 = id % plan.tiles;
    id /= plan.tiles;
    const int head = id % a.Hkv, s = id / a.Hkv;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, h = lane / 16, r16 = lane % 16;
    const Seq seq = seq_of(a, s);
    const int rows = seq.count * a.group, page_mask = (1 << a.page_shift) - 1;
    const T *kc = (const T *)a.k + head * a.cache.head, *vc = (const T *)a.v + head * a.cache.head;

    // max_q sets the grid; a sequence with more new tokens goes round again
    for (int r0 = tile0 * ROWS; r0 < rows; r0 += plan.tiles * ROWS) {
        const Span sp = span_of_rows(a, seq, r0, ROWS);
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
        const int first = seq.len - seq.count + r0 / a.group, last = sp.end - 1;
        bool bad = seq.cut;

        for (int i0 = begin + 2 * wave; i0 < end; i0 += 2 * WAVES) {
            typename M::K k[2];
            typename M::V v;
            int base[2];
            bool all = i0 + 1 < end;   // every row sees every key of the step
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int tile = sp.tile(min(i0 + i, end - 1));
                const int n0 = tile * KT;
                base[i] = i0 + i < end ? n0 : INT32_MAX - KT;   // past every position
                all &= n0 + KT - 1 <= first && (n0 > last - a.window || n0 + KT <= a.sinks);
                int page = a.table[(size_t)s * a.table_cols + (n0 >> a.page_shift)];
                if ((unsigned)page >= (unsigned)a.pages) {
                    bad = true;
                    page = 0;
                }
                const int nk = sp.read(n0 + r16, n0 + KT - 1);
                const T *kp = kc + page * a.cache.batch, *vp = vc + page * a.cache.batch;
                M::ld_row(kp + (nk & page_mask) * a.cache.token, h, k[i].x);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int nv = sp.read(n0 + 4 * h + j, n0 + KT - 1);
                    M::ld_v(vp + (nv & page_mask) * a.cache.token, r16, v.x[4 * i + j]);
                }
            }
            // A value that is infinite or NaN takes the step out of MFMA: a row
            // whose weight is 0 because it does not see the key would get NaN,
            // and so would infinity times a weight's second part.
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
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    for (int hh = 0; hh < 4; ++hh) {
                        const float wk = __shfl(w[i / 4][i % 4], 16 * hh + r16);
                        const int n = base[i / 4] + 4 * hh + i % 4;
                        if (!visible(n, pos[r], a.window, a.sinks)) continue;
                        const int page = a.table[(size_t)s * a.table_cols + (n >> a.page_shift)];
                        if ((unsigned)page >= (unsigned)a.pages) continue;
                        const T *vp = vc + page * a.cache.batch + (n & page_mask) * a.cache.token + h * (D / 4);
#pragma unroll
                        for (int d = 0; d < D / 4; ++d)
                            acc[r][d % VW][d / VW] = fmaf(wk, io<T>::ld(vp, d), acc[r][d % VW][d / VW]);
                    }
                }
            }
        }

        // the waves' sums, one row tile at a time
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            __syncthreads();
            const float gs = rows4_sum(g[r]);
            if (h == 0) gred[wave][r16] = bad ? __builtin_nanf("") : gs;
#pragma unroll
            for (int d = 0; d < D / 4; ++d) red[wave][r16][h * (D / 4) + d] = acc[r][d % VW][d / VW];
            __syncthreads();
            const int rr = threadIdx.x / 16, c = threadIdx.x % 16 * VW, row = r0 + 16 * r + rr;
            if (row < rows) {
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

// Adds the splits' sums: 16 lanes a row.
template <typename T, int D>
__global__ __launch_bounds__(THREADS) void join_kernel(PagedArgs a, PagedPlan plan, const float *part)
{
    constexpr int VW = D / 16;
    const int s = blockIdx.y;
    const Seq seq = seq_of(a, s);
    const long long n = (long long)seq.count * a.Hq;
    const int c = threadIdx.x % 16 * VW;
    const float *gpart = part + (size_t)a.T * a.Hq * plan.splits * D;
    for (long long i = (long long)blockIdx.x * (THREADS / 16) + threadIdx.x / 16; i < n;
         i += (long long)gridDim.x * (THREADS / 16)) {
        const int t = (int)(i / a.Hq), head = (int)(i - (long long)t * a.Hq);
        const int row = t * a.group + head % a.group, rows = 16 * plan.row_tiles;
        const Span sp = span_of_rows(a, seq, row / rows * rows, rows);
        const int used = max(1, min(plan.splits, (sp.tiles + plan.chunk - 1) / plan.chunk));
        const size_t o = (size_t)(seq.t0 + t) * a.Hq + head;
        float f[VW], g = 0.f;
#pragma unroll
        for (int j = 0; j < VW; ++j) f[j] = 0.f;
        for (int k = 0; k < used; ++k) {
            const float *p = part + (o * plan.splits + k) * D + c;
            g += gpart[o * plan.splits + k];
#pragma unroll
            for (int j = 0; j < VW; ++j) f[j] += p[j];
        }
        const bool none = seq.len - seq.count + t < 0;
        T *out = (T *)a.out + o * D + c;
#pragma unroll
        for (int j = 0; j < VW; ++j) io<T>::st(out, j, none ? 0.f : f[j] / g);
    }
}

template <typename T, int D, int RT>
hipError_t launch(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    const long long blocks = (long long)plan.splits * plan.tiles * a.Hkv * a.S;
    if (!grid_fits(blocks, THREADS) || a.S > 65535) return hipErrorInvalidConfiguration;
    if (a.q_start) paged_kernel<T, D, RT, true><<<(unsigned)blocks, THREADS, 0, st>>>(a, plan, part);
    else paged_kernel<T, D, RT, false><<<(unsigned)blocks, THREADS, 0, st>>>(a, plan, part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.splits == 1) return e;
    const int rows = 16 * RT * plan.tiles / a.group * a.Hq;
    const dim3 grid((unsigned)((rows + 15) / 16), (unsigned)a.S);
    join_kernel<T, D><<<grid, THREADS, 0, st>>>(a, plan, part);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_rt(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    switch (plan.row_tiles) {
    case 1: return launch<T, D, 1>(a, plan, part, st);
    case 2: return launch<T, D, 2>(a, plan, part, st);
    default: return launch<T, D, 4>(a, plan, part, st);
    }
}

template <typename T> hipError_t launch_d(const PagedArgs &a, const PagedPlan &plan, int D, float *part, hipStream_t st)
{
    switch (D) {
    case 16: return launch_rt<T, 16>(a, plan, part, st);
    case 32: return launch_rt<T, 32>(a, plan, part, st);
    case 64: return launch_rt<T, 64>(a, plan, part, st);
    default: return launch_rt<T, 128>(a, plan, part, st);
    }
}

}  // namespace

PagedPlan paged_plan(int S, int Hq, int Hkv, int D, int is_bf16, int max_q, int max_len, int window,
                     int sinks)
{
    PagedPlan plan;
    const long long rows = (long long)max_q * (Hq / Hkv);
    plan.row_tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const long long per = 16 * plan.row_tiles, tiles = (rows + per - 1) / per;
    // the most key tiles that a row tile can see
    const long long tokens = per * Hkv / Hq + 2;
    const long long seen = (long long)window + tokens + 2 * KT + sinks;
    const long long keys = max_len < seen ? max_len : seen;
    const long long key_tiles = (keys + KT - 1) / KT;
    // about 1024 workgroups, 256 keys in each at least
    const long long base = tiles * Hkv * S;
    long long splits = (1024 + base - 1) / base;
    const long long most = (key_tiles + 15) / 16;
    splits = splits < most ? splits : most;
    long long chunk = (key_tiles + splits - 1) / splits;
    chunk = (chunk + 2 * WAVES - 1) / (2 * WAVES) * (2 * WAVES);
    plan.tiles = (int)(tiles < INT32_MAX ? tiles : INT32_MAX);
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
