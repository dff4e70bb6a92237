// Fastmax attention of new tokens over a paged cache of 8-bit rows: key n is
// ks_n c_n, value n is vs_n e_n with codes c_n, e_n of -127 .. 127 and a float32
// scale each (fm_paged.hip has the formulas and what a row sees).
//
// A code is always a number, so what unseen slots hold needs no care beyond their
// scales, which a select keeps out.
//
// Few rows (single tokens).  HBM bounds it, D + 4 bytes a row: 4.8 TB/s at even
// lengths, 61 sequences of up to 8192 tokens, 32 heads to 8 of 128, 100 us (3.8 TB/s,
// the longest end alone), float32 102.  A wave walks over key tiles of 16, two at a time, straight
// from the cache into registers, as fm_paged.hip.  Scores take the codes as they are:
// q^ of a row becomes one 16-bit (float32: 24-bit) whole number per channel under a
// scale of its row, cut in signed bytes, and int8 MFMA gives exact sums,
//     q^ = qs (256 a + b)  ->  s = qs ks (256 a.c + b.c),
// two products of int8 at the price of one in bf16 and no conversion of keys; q^ is off
// by at most 2^-16 (2^-23) of the row's largest magnitude.  Values: weights times vs in
// two bf16 parts (float32: three) against the codes, which bf16 holds exactly.
//
// Many rows (chunks).  The matrix pipe and the instructions beside it bound it: four
// chunks of up to 2048 tokens over up to 8192, 32 heads to 8 of 128, 456 to 545 us, 650
// TFLOP/s and more (cards differ); float32, with twice the products, 855.  There the few rows' scheme took 766: each wave converted every code for
// itself, and weights entered as two parts.  So codes become fp16 once a workgroup, on
// their way into LDS, and one fp16 product (11 bits) does for weights and scores.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "fm_internal.h"
#include "fm_paged.h"
#include "fm_pairs_rows.h"
#include "fm_rows.h"
#include "fm_serve.h"

namespace fm {
namespace {

using namespace paged;

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i16v __attribute__((ext_vector_type(16)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int WAVES = 4, THREADS = 64 * WAVES;

// Bytes of a whole number of q^, and bf16 parts of a weight.
template <typename T> constexpr int PARTS = sizeof(T) == 2 ? 2 : 3;

// Largest over the four rows of 16 lanes, in every lane.
__device__ __forceinline__ uint32_t rows4_max(uint32_t x)
{
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(b[0], b[1]);
}
__device__ __forceinline__ uint32_t halves_max(uint32_t x)
{
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max(b[0], b[1]);
}
__device__ __forceinline__ float halves_sum(float x)
{
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <int N> __device__ __forceinline__ uint32_t abs_max(const float *x)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    return top;
}

// A row's whole numbers: the factor from its values, and the scale back.  The
// largest magnitude (float32 bits) becomes M, whose bytes are at most 127 (24
// bits: with room for the product's rounding).  A row that is not finite has no
// numbers (NaN); below 2^-100 it is 0.
template <int NP> __device__ __forceinline__ float2 whole_scale(uint32_t top)
{
    constexpr float M = NP == 2 ? 32639.0f : 8355584.0f;
    const float amax = __uint_as_float(top);
    if (top >= 0x7f800000u) return make_float2(0.f, __builtin_nanf(""));
    if (amax < Q8_LEAST) return make_float2(0.f, 0.f);
    return make_float2(M / amax, amax / M);
}

// Four values as whole numbers, byte p of each in word p (the highest first).
template <int NP> __device__ __forceinline__ void whole4(const float *x, float f, uint32_t *w)
{
#pragma unroll
    for (int p = 0; p < NP; ++p) w[p] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y = x[i] * f;
        int n = y == y ? __float2int_rn(y) : 0;
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) {
            const int b = (int)(int8_t)n;
            w[p] |= (uint32_t)(b & 255) << (8 * i);
            n = (n - b) >> 8;
        }
    }
}

// Byte j of two words as two bf16 (whole numbers up to 127 have few bits).
__device__ __forceinline__ uint32_t codes2(uint32_t a, uint32_t b, int j)
{
    const float x = (float)(int8_t)(a >> (8 * j)), y = (float)(int8_t)(b >> (8 * j));
    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}

// Two weights as NP pairs of bf16 parts, each the rest of the ones before it.
template <int NP> __device__ __forceinline__ void parts2(float x, float y, uint32_t *p)
{
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        p[i] = rows::pack2(x, y);
        x -= __uint_as_float(p[i] << 16);
        y -= __uint_as_float(p[i] & 0xffff0000u);
    }
}

template <int N, typename T> __device__ __forceinline__ void ld_row(const T *p, float *x)
{
#pragma unroll
    for (int i = 0; i < N; i += 8) rows::ld8(p + i, x + i);
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

// --- few rows -------------------------------------------------------------------

// 16x16x64 int8 (D >= 64: a lane of row h holds channels 64 c + 16 h .. + 15) or
// 16x16x32 (channels 8 h .. 8 h + 7; D = 16: rows 0 and 1 only).
template <typename T, int D> struct Few {
    static constexpr int NP = PARTS<T>;
    static constexpr int QC = D >= 64 ? D / 64 : 1, QB = D >= 64 ? 16 : 8;   // pieces, bytes of one
    static constexpr int VW = D / 16;
    struct Q { u4 x[NP][QC]; float scale; };
    struct K { u4 x[QC]; };
    struct V { uint32_t x[8][VW > 4 ? 2 : 1]; };

    static __device__ __forceinline__ void ld_q(const T *p, int h, Q &q)
    {
        float x[QC][QB];
        uint32_t top = 0;
        const bool in = D >= 32 || h < 2;
#pragma unroll
        for (int c = 0; c < QC; ++c) {
            ld_row<QB>(p + (in ? 64 * c + QB * h : 0), x[c]);
            top = max(top, abs_max<QB>(x[c]));
        }
        const float2 f = whole_scale<NP>(rows4_max(top));
        q.scale = f.y;
#pragma unroll
        for (int c = 0; c < QC; ++c) {
#pragma unroll
            for (int i = 0; i < QB / 4; ++i) {
                uint32_t w[NP];
                whole4<NP>(x[c] + 4 * i, f.x, w);
#pragma unroll
                for (int n = 0; n < NP; ++n) q.x[n][c][i] = in ? w[n] : 0u;
            }
        }
    }
    static __device__ __forceinline__ void ld_k(const int8_t *p, int h, K &k)
    {
        if constexpr (D >= 64) {
#pragma unroll
            for (int c = 0; c < QC; ++c) k.x[c] = *(const u4 *)(p + 64 * c + 16 * h);
        } else {
            // D = 16: the queries' bytes are 0 where h > 1
            const uint2 u = *(const uint2 *)(p + (D == 16 ? h & 1 : h) * 8);
            k.x[0] = u4{u.x, u.y, 0, 0};
        }
    }
    static __device__ __forceinline__ i4 mma(const K &k, const u4 *q, i4 s)
    {
#pragma unroll
        for (int c = 0; c < QC; ++c) {
            if constexpr (D >= 64) {
                s = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i4, k.x[c]), __builtin_bit_cast(i4, q[c]),
                                                          s, 0, 0, 0);
            } else {
                const uint2 a = make_uint2(k.x[c][0], k.x[c][1]), b = make_uint2(q[c][0], q[c][1]);
                s = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), s,
                                                          0, 0, 0);
            }
        }
        return s;
    }
    // Sums of products of the whole numbers: |256 a.c + b.c| < 2^30.
    static __device__ __forceinline__ f4 scores(const K &k, const Q &q)
    {
        const i4 z = {0, 0, 0, 0};
        const i4 s = mma(k, q.x[1], mma(k, q.x[0], z) << 8);
        f4 r;
        if constexpr (NP == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = (float)s[i];
        } else {
            const i4 l = mma(k, q.x[2], z);
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = fmaf((float)s[i], 256.0f, (float)l[i]);
        }
        return r;
    }
    // key i of the lane's eight: tile i / 4, key 4 h + i % 4
    static __device__ __forceinline__ void ld_v(const int8_t *p, int r16, uint32_t *x)
    {
        p += r16 * VW;
        if constexpr (VW == 8) {
            const uint2 u = *(const uint2 *)p;
            x[0] = u.x; x[1] = u.y;
        } else if constexpr (VW == 4) {
            x[0] = *(const uint32_t *)p;
        } else if constexpr (VW == 2) {
            x[0] = *(const uint16_t *)p;
        } else {
            x[0] = *(const uint8_t *)p;
        }
    }
    // acc[j] += V^T W^T for channel r16 VW + j
    static __device__ __forceinline__ void add(f4 *acc, const V &v, const f4 *w)
    {
        u4 b[NP];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t p[NP];
            parts2<NP>(w[i / 2][2 * (i % 2)], w[i / 2][2 * (i % 2) + 1], p);
#pragma unroll
            for (int n = 0; n < NP; ++n) b[n][i] = p[n];
        }
#pragma unroll
        for (int j = 0; j < VW; ++j) {
            u4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = codes2(v.x[2 * i][j / 4], v.x[2 * i + 1][j / 4], j % 4);
#pragma unroll
            for (int n = NP - 1; n >= 0; --n)
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, x), __builtin_bit_cast(b8, b[n]),
                                                                 acc[j], 0, 0, 0);
        }
    }
};

// At D = 128 registers are bounded for three waves on a SIMD: 61 sequences of 4096
// keys, 8 heads 110 us, 117 with the two that it takes unbounded, 127 with four.
template <typename T, int D, int RT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, RT == 1 && WAVES == 4 && D == 128 ? 3 : 1) void few_kernel(PagedArgs a, PagedPlan plan, float *part)
{
    using M = Few<T, D>;
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
    const int8_t *kc = (const int8_t *)a.k + head * a.cache.head, *vc = (const int8_t *)a.v + head * a.cache.head;
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
        float c1[RT], c2[RT], g[RT];
        f4 acc[RT][VW];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = min(r0 + 16 * r + r16, rows - 1);
            const int t = row / a.group;
            pos[r] = seq.len - seq.count + t;
            M::ld_q((const T *)a.q + (seq.t0 + t) * a.q_token + (head * a.group + row - t * a.group) * a.q_head, h, q[r]);
            c1[r] = a.c1 * q[r].scale;
            c2[r] = a.c2 * q[r].scale * q[r].scale;
            g[r] = 0.f;
#pragma unroll
            for (int j = 0; j < VW; ++j) acc[r][j] = f4{0.f, 0.f, 0.f, 0.f};
        }
        const int first = scalar(seq.len - seq.count + r0 / a.group), last = sp.end - 1;
        // Key tiles [whole, whole_end) exist in full and every row sees all their
        // keys; elsewhere weights are masked.
        const int shift = sp.low - sp.sink_tiles;   // from a tile's number here to its own
        const int whole = a.window < sp.end ? max(sp.sink_tiles, (last - a.window) / KT + 1 - shift) : 0;
        const int whole_end = min(end, (first + 1) / KT - shift);
        bool bad = seq.cut;

        // The wave's steps of two key tiles, 32 steps at a time, their pages a
        // tile to a lane, so that no step waits for the page table.
        for (int b0 = begin + 2 * wave; b0 < end; b0 += 64 * WAVES) {
            const int mine = sp.tile(min(b0 + lane / 2 * (2 * WAVES) + lane % 2, end - 1)) * KT;
            int page = table[mine >> a.page_shift];
            if ((unsigned)page >= (unsigned)a.pages) {
                bad = true;
                page = 0;
            }
            for (int n = 0; n < 32; ++n) {
                const int i0 = b0 + n * (2 * WAVES);
                if (i0 >= end) break;
                typename M::K k[2];
                typename M::V v;
                f4 ks[2], vs[2];
                const bool all = i0 >= whole && i0 + 2 <= whole_end;
                int base[2];   // of the key tiles; past every position if there is none
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const long long pg = __builtin_amdgcn_readlane(page, 2 * n + i);
                    const int n0 = sp.tile(min(i0 + i, end - 1)) * KT, place = n0 & page_mask;
                    const long long from = pg * a.cache.batch + place * a.cache.token;
                    const long long at = ((pg * a.Hkv + head) << a.page_shift) + place;
                    base[i] = i0 + i < end ? n0 : INT32_MAX - KT;
                    M::ld_k(kc + from + r16 * token, h, k[i]);
                    ks[i] = *(const f4 *)(a.k_scale + at + 4 * h);
                    vs[i] = *(const f4 *)(a.v_scale + at + 4 * h);
#pragma unroll
                    for (int j = 0; j < 4; ++j) M::ld_v(vc + from + (4 * h + j) * token, r16, v.x[4 * i + j]);
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    f4 w[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const f4 x = M::scores(k[i], q[r]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float y = x[j] * ks[i][j];
                            float f = fmaf(fmaf(y, c2[r], c1[r]), y, 1.0f), fv = f * vs[i][j];
                            if (!all && !visible(base[i] + 4 * h + j, pos[r], a.window, a.sinks)) f = fv = 0.f;
                            g[r] += f;
                            w[i][j] = fv;
                        }
                    }
                    M::add(acc[r], v, w);
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

template <typename T, int D, int RT, int W = WAVES>
hipError_t launch_few(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    const long long blocks = (long long)plan.splits * plan.tiles * a.Hkv * a.S;
    if (!grid_fits(blocks, 64 * W)) return hipErrorInvalidConfiguration;
    few_kernel<T, D, RT, W><<<(unsigned)blocks, 64 * W, 0, st>>>(a, plan, part);
    return hipGetLastError();
}

// --- many rows ------------------------------------------------------------------

// LDS rows have no padding: piece c of row r (16 bytes) lies at c ^ swizzle(r),
// which puts 8 consecutive rows' piece c, and pieces c, c + 1 of 4 consecutive
// rows, on distinct banks.
template <int C> __device__ __forceinline__ int swizzle(int r)
{
    if constexpr (C >= 8) return (r & 3) << 1 | (r >> 2 & 1);
    else return (r >> 1 & 1) << 1 | (r >> 2 & 1);   // two rows to a line of banks
}

// Four codes as fp16, exactly: 1024 + (128 + code) by its bits, then less 1152.
__device__ __forceinline__ uint2 codes4(uint32_t w)
{
    const pr::h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    w ^= 0x80808080u;
    const uint32_t lo = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u), hi = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u);
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_bit_cast(pr::h2, lo) - off),
                      __builtin_bit_cast(uint32_t, __builtin_bit_cast(pr::h2, hi) - off));
}

// Products with fp16 operands of FP parts (bf16 calls: one; float32: two, each the
// rest of the one before it).  128 rows to a workgroup, 32 to a wave, 64 keys at a
// time through two LDS buffers, products of 32x32 as fm_paged_chunk.hip (its
// layouts: lane = 32 hh + c32; accumulator register i: column c32, row 8 (i/4) + 4 hh
// + i%4).  The cache's bytes go through registers, where a workgroup turns its codes
// into fp16 once for its four waves.
//
// Powers of two keep fp16's range.  A row of q is taken times one of its own (bf16
// rows stay exact but for what is 2^-17 of their largest); weights times 2^-e, which
// costs nothing in 1 + x (c1 + c2 x): with |k_n| <= 127 sqrt(D) ks_n a row's largest
// possible weight stays below 2^14; values times 2^-P.  e and P follow from the largest
// scales that a row has seen so far (P, where every row sees the whole step, from the
// wave's): a wave that meets a larger one scales its sums.
// What it takes per pair beside the products: ks x, the weight (2), its conversion,
// sum and scale in packed halves (4.5 instructions in bf16).
template <typename T, int D>
__global__ __launch_bounds__(THREADS, sizeof(T) == 4 && D == 128 ? 1 : 2) void many_kernel(PagedArgs a, PagedPlan plan, int pieces, float *part)
{
    constexpr int FP = sizeof(T) == 2 ? 1 : 2, ROWS = CHUNK_ROWS, WR = ROWS / 4, KB = 64, STEP = KB / KT;
    constexpr int C = D / 8, KS = D / 16, DT = D / 32;        // 16-byte pieces of a row, score steps, channel tiles
    constexpr int LP = D / 16;                                // 16-byte loads of a row of codes
    constexpr int LN = KT * LP > 64 ? KT * LP / 64 : 1, LR = 64 / LP;   // loads of a lane, rows of one
    static_assert(STEP == THREADS / 64, "a wave loads a key tile of a step");
    __shared__ u4 keys0[KB * C], keys1[KB * C], values0[KB * C], values1[KB * C];
    __shared__ f4 kscale[2][KB / 4], vscale[2][KB / 4];
    __shared__ f4 factors[THREADS / 64][KB / 4];              // of values in whole steps, a wave's own (bf16: halves)

    // Row tiles of one (sequence, key head, split) read the same keys, so every
    // `pieces`th of them go to the same XCD.  Late row tiles see the most keys and
    // start first.
    const int in_piece = (plan.tiles + pieces - 1) / pieces;
    const int turn = blockIdx.x / 8 / in_piece, piece = turn * 8 + (blockIdx.x + turn) % 8;
    const int row_tile = plan.tiles - 1 - (piece % pieces + pieces * (blockIdx.x / 8 % in_piece));
    const int split = piece / pieces % plan.splits, pair = piece / pieces / plan.splits;
    if (pair >= a.S * a.Hkv || row_tile < 0) return;
    const int head = pair % a.Hkv, s = pair / a.Hkv;

    const int wave = scalar(threadIdx.x / 64), lane = threadIdx.x % 64, hh = lane / 32, c32 = lane % 32;
    const Seq seq = seq_of(a, s);
    const int rows = seq.count * a.group, page_mask = (1 << a.page_shift) - 1;
    const int8_t *kc = (const int8_t *)a.k + head * a.cache.head, *vc = (const int8_t *)a.v + head * a.cache.head;
    const int32_t *table = a.table + (size_t)s * a.table_cols;
    // A wave loads one key tile of a step, whose page is a scalar: a lane's place in it
    // does not change.  (Places and pages by lane, for 64 rows shared out evenly: 603 us
    // where this takes 541.)
    const int my_row = KT * wave + lane / LP, my_piece = lane % LP;
    const bool loads = KT * LP >= 64 || lane < KT * LP;
    const int token = (int)a.cache.token, my_at = lane / LP * token + 16 * my_piece;
    const float *const my_scale = (lane < KT ? a.k_scale : a.v_scale) + lane % KT;

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
        u4 q[FP][KS];
        float size;          // the row's norm times tau 127 sqrt(D): |s| < size ks
        float qs;            // the row's power of two; NaN: the row is not finite
        {
            const T *p = (const T *)a.q + (seq.t0 + t) * a.q_token + q_head * a.q_head + 8 * hh;
            float x[KS][8], ss = 0.f;
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                rows::ld8(p + 16 * k, x[k]);
                top = max(top, abs_max<8>(x[k]));
            }
            top = halves_max(top);
            const bool odd = top >= 0x7f800000u;
            const int e = odd || top == 0 ? 0 : (int)(top >> 23) - 126;   // |x| < 2^e
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                pr::h2 hi[4], lo[4];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[k][i] = __builtin_ldexpf(x[k][i], 10 - e);
                    ss = fmaf(x[k][i], x[k][i], ss);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    hi[i] = pr::cvt2(x[k][2 * i], x[k][2 * i + 1]);
                    lo[i] = pr::cvt2(pr::rest(x[k][2 * i], hi[i][0]), pr::rest(x[k][2 * i + 1], hi[i][1]));
                    q[0][k][i] = __builtin_bit_cast(uint32_t, hi[i]);
                    if constexpr (FP == 2) q[1][k][i] = __builtin_bit_cast(uint32_t, lo[i]);
                }
            }
            qs = odd ? __builtin_nanf("") : __builtin_ldexpf(1.0f, e - 10);
            size = odd ? 0.f : a.c1 * __builtin_ldexpf(sqrtf(halves_sum(ss)) * (130.0f * sqrtf((float)D)), e - 10);
        }
        f16v acc[DT];
        float g = 0.f, c0 = 1.f, c1 = 0.f, c2 = 0.f;   // weight c0 + x (c1 + c2 x), times 2^-e
        int kpower = -1000, vpower = -1000, e = 0;     // the largest of the scales seen so far; e: see c0
        int all_k = 0, all_v = 0;                      // in whole steps: the least kpower, the wave's vpower
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] = f16v{};

        bool bad = seq.cut;
        // Key tiles [whole, whole_end) exist in full and every row sees all their
        // keys; elsewhere weights are masked.
        const int shift = sp.low - sp.sink_tiles;   // from a tile's number here to its own
        const int whole = a.window < sp.end ? max(sp.sink_tiles, (last - a.window) / KT + 1 - shift) : 0;
        const int whole_end = min(end, (first + 1) / KT - shift);

        // A step's bytes in registers: this lane's pieces of keys and values, and a
        // scale (lanes 0 .. 15: of a key, 16 .. 31: of a value).
        u4 kr[LN], vr[LN];
        float sr = 0.f;
        const auto tile_of = [&](int i0) { return scalar(sp.tile(min(i0 + wave, end - 1)) * KT); };
        int page = 0;   // of the next load's tile, a step ahead
        const auto page_of = [&](int i0) { page = table[tile_of(i0) >> a.page_shift]; };
        const auto load = [&](int i0) {
            const int place = tile_of(i0) & page_mask;
            int pg = scalar(page);
            if ((unsigned)pg >= (unsigned)a.pages) {
                bad = true;
                pg = 0;
            }
            const long long at = pg * a.cache.batch + place * a.cache.token;
            if (loads) {
#pragma unroll
                for (int i = 0; i < LN; ++i) {
                    kr[i] = *(const u4 *)(kc + at + (my_at + LR * i * token));
                    vr[i] = *(const u4 *)(vc + at + (my_at + LR * i * token));
                }
            }
            if (lane < 2 * KT) sr = my_scale[(((long long)pg * a.Hkv + head) << a.page_shift) + place];
        };
        const auto store = [&](u4 *k, u4 *v, int b) {
            if (loads) {
#pragma unroll
                for (int i = 0; i < LN; ++i) {
                    const int r = my_row + LR * i;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int to = r * C + ((2 * my_piece + j) ^ swizzle<C>(r));
                        const uint2 k0 = codes4(kr[i][2 * j]), k1 = codes4(kr[i][2 * j + 1]);
                        const uint2 v0 = codes4(vr[i][2 * j]), v1 = codes4(vr[i][2 * j + 1]);
                        k[to] = u4{k0.x, k0.y, k1.x, k1.y};
                        v[to] = u4{v0.x, v0.y, v1.x, v1.y};
                    }
                }
            }
            if (lane < 2 * KT) ((float *)(lane < KT ? kscale : vscale)[b])[KT * wave + lane % KT] = sr;
        };

        // Which of keys {0 .. 3} + 8 i + 4 hh of 32 the lane's row sees: key n0 + n of a
        // tile if n <= lim and (n > lim - window or it is a first token).
        struct Limits { int lim, low, sinks; };
        const auto limits = [&](int i0, int kb, int i) {
            const int it = i0 + 2 * kb + i / 2, n0 = sp.tile(min(it, end - 1)) * KT + 4 * hh;
            const int lim = it < end ? max(pos, -1) - n0 : -1;
            return Limits{lim, lim - a.window, a.sinks - n0};
        };
        const auto sees = [&](const Limits &l, int n) { return n <= l.lim && (n > l.low || n < l.sinks); };
        // The step's powers, and its values' factors.
        const auto raise = [&](int pk, int from, int v) {
            kpower = max(kpower, pk);
            const float most = __builtin_ldexpf(size, kpower);
            const float w = a.c2 == 0.f ? 1.0f + most : fmaf(0.5f * most, most, 1.0f + most);
            const int to = w < 3e38f ? pr::exp_above(w) - 14 : 114;
            const float fg = __builtin_ldexpf(1.0f, max(e - to, -300)), f = __builtin_ldexpf(fg, max(from - v, -300));
            g *= fg;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[d] *= f;
            e = to;
            c0 = __builtin_ldexpf(1.0f, -e);
            c1 = a.c1 * qs * c0;
            c2 = a.c2 * qs * (qs * c0);
        };
        const auto powers = [&](int b, int i0, auto masked) {
            if constexpr (decltype(masked)::value) {
                // by step, then, if that is more than a row's so far, by what each row sees
                // (what none sees may be anything)
                const float ks = ((const float *)kscale[b])[lane], vs = ((const float *)vscale[b])[lane];
                const int pk = wave_max(pr::exp_above(fabsf(ks))), pv = wave_max(pr::exp_above(fabsf(vs)));
                if (__any(pk > kpower || pv > vpower)) {
                    uint32_t k = 0, v = 0;
#pragma unroll 1
                    for (int j = 0; j < KB / 8; ++j) {
                        const f4 k4 = kscale[b][2 * j + hh], v4 = vscale[b][2 * j + hh];
                        const Limits l = limits(i0, j / 4, j % 4);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t x = __float_as_uint(fabsf(k4[i])), y = __float_as_uint(fabsf(v4[i]));
                            const bool see = sees(l, 8 * (j % 2) + i);
                            k = see && x < 0x7f800000u ? max(k, x) : k;
                            v = see && y < 0x7f800000u ? max(v, y) : v;
                        }
                    }
                    const int seen_k = pr::exp_above(__uint_as_float(halves_max(k))),
                              seen_v = pr::exp_above(__uint_as_float(halves_max(v)));
                    const int to = max(vpower, seen_v);
                    raise(seen_k, vpower, to);
                    vpower = to;
                }
            } else {
                const float ks = ((const float *)kscale[b])[lane], vs = ((const float *)vscale[b])[lane];
                int pk = pr::exp_above(fabsf(ks)), pv = pr::exp_above(fabsf(vs));
                if (__any(pk > all_k || pv > all_v)) {
                    pk = wave_max(pk);
                    pv = wave_max(pv);
                    raise(pk, all_v, max(all_v, pv));
                    all_k = max(all_k, pk);
                    all_v = max(all_v, pv);
                }
                const float f = __builtin_ldexpf(vs, -all_v);
                if constexpr (FP == 1) ((_Float16 *)factors[wave])[lane] = (_Float16)f;
                else ((float *)factors[wave])[lane] = f;
            }
        };
        const auto scores = [&](const u4 *kt, int kb) {
            u4 k[KS];
#pragma unroll
            for (int i = 0; i < KS; ++i) k[i] = kt[(32 * kb + c32) * C + ((2 * i + hh) ^ swizzle<C>(c32))];
            f16v x = f16v{};
#pragma unroll
            for (int n = FP - 1; n >= 0; --n)
#pragma unroll
                for (int i = 0; i < KS; ++i)
                    x = pr::mma(__builtin_bit_cast(pr::h8, k[i]), __builtin_bit_cast(pr::h8, q[n][i]), x);
            return x;
        };
        const auto block = [&](const f16v &x, const u4 *vt, int b, int i0, int kb, auto masked) {
            u4 va[2][DT];
            // the value operands: keys {4 hh .. + 3, 8 + 4 hh .. + 3} of 16, channel c32 of 32
            const s4 *v = (const s4 *)vt;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    typedef s4 __attribute__((address_space(3))) *lp;
                    const int j = lane >> 2 & 3, r = 32 * kb + 16 * m + 4 * hh + j;
                    const int c = 4 * d + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
                    const int at = 2 * (r * C + (c ^ swizzle<C>(4 * hh + j))) + (lane & 1);
                    const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(v + at));
                    const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(v + at + 2 * 8 * C));
                    const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
                    va[m][d] = u4{l.x, l.y, h.x, h.y};
                }
            }
            u4 w[FP][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f4 ks = kscale[b][8 * kb + 2 * i + hh];
                float y[4];
                f4 f;
                pr::h2 fh[2];
                Limits l;
                if constexpr (decltype(masked)::value) {
                    f = vscale[b][8 * kb + 2 * i + hh];
                    l = limits(i0, kb, i);
                } else if constexpr (FP == 1) {
                    const h4 x = ((const h4 *)factors[wave])[8 * kb + 2 * i + hh];
                    fh[0] = pr::h2{x[0], x[1]};
                    fh[1] = pr::h2{x[2], x[3]};
                } else {
                    f = factors[wave][8 * kb + 2 * i + hh];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float z = x[4 * i + j] * ks[j];
                    y[j] = fmaf(fmaf(z, c2, c1), z, c0);
                    if constexpr (decltype(masked)::value) {
                        const bool see = sees(l, 8 * (i % 2) + j);
                        y[j] = see ? y[j] : 0.f;
                        f[j] = see ? __builtin_ldexpf(f[j], -vpower) : 0.f;
                    }
                }
                if constexpr (FP == 1 && decltype(masked)::value) {
                    fh[0] = pr::cvt2(f[0], f[1]);
                    fh[1] = pr::cvt2(f[2], f[3]);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if constexpr (FP == 1) {
                        // the sum of the rounded weights, as the numerator takes them
                        const pr::h2 one = {(_Float16)1.0f, (_Float16)1.0f};
                        const pr::h2 h = pr::cvt2(y[2 * j], y[2 * j + 1]);
                        g = __builtin_amdgcn_fdot2(h, one, g, false);
                        const pr::h2 o = h * fh[j];
                        w[0][i / 2][2 * (i % 2) + j] = __builtin_bit_cast(uint32_t, o);
                    } else {
                        g += y[2 * j] + y[2 * j + 1];
                        float z[2];
#pragma unroll
                        for (int n = 0; n < 2; ++n) z[n] = y[2 * j + n] * f[2 * j + n];
                        const pr::h2 hi = pr::cvt2(z[0], z[1]), lo = pr::cvt2(pr::rest(z[0], hi[0]), pr::rest(z[1], hi[1]));
                        w[0][i / 2][2 * (i % 2) + j] = __builtin_bit_cast(uint32_t, hi);
                        w[FP - 1][i / 2][2 * (i % 2) + j] = __builtin_bit_cast(uint32_t, lo);
                    }
                }
            }
#pragma unroll
            for (int n = FP - 1; n >= 0; --n)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int d = 0; d < DT; ++d)
                        acc[d] = pr::mma(__builtin_bit_cast(pr::h8, va[m][d]), __builtin_bit_cast(pr::h8, w[n][m]), acc[d]);
        };
        // (loops of their own for whole and for masked steps: one loop for both moves the
        // sums between registers)
        const auto walk = [&](u4 *__restrict__ k0, u4 *__restrict__ k1, u4 *__restrict__ v0, u4 *__restrict__ v1) {
            if (begin < end) {
                page_of(begin);
                load(begin);
                page_of(begin + STEP);
                store(k0, v0, 0);
                load(begin + STEP);
                page_of(begin + 2 * STEP);
            }
            __syncthreads();
            const auto turn = [&](u4 *k, u4 *v, int b, int i0) {
                // the other buffer: every wave is past the step that read it
                store(k, v, b);
                load(i0 + 2 * STEP);
                page_of(i0 + 3 * STEP);
                __syncthreads();
            };
            const auto pairs = [&](int i0, int to, auto masked) {
                const auto step = [&](const u4 *k, const u4 *v, int b, int i) {
                    powers(b, i, masked);
#pragma unroll
                    for (int kb = 0; kb < KB / 32; ++kb) block(scores(k, kb), v, b, i, kb, masked);
                };
                for (; i0 < to; i0 += 2 * STEP) {
                    step(k0, v0, 0, i0);
                    turn(k1, v1, 1, i0);
                    if (i0 + STEP >= end) return;
                    step(k1, v1, 1, i0 + STEP);
                    turn(k0, v0, 0, i0 + STEP);
                }
            };
            const int from = min(begin + max(whole - begin + 2 * STEP - 1, 0) / (2 * STEP) * (2 * STEP), end);
            const int to = max(from, begin + max(whole_end - begin, 0) / (2 * STEP) * (2 * STEP));
            pairs(begin, from, std::true_type{});
            if (from < min(to, end)) {
                // values by one power for the wave: the least of the rows', which keeps all
                // their bits (within 2^80, for what the sums have room for)
                all_v = max(-wave_max(-vpower), wave_max(vpower) - 80);
                all_k = -wave_max(-kpower);
                const float f = __builtin_ldexpf(1.0f, max(vpower - all_v, -300));
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[d] *= f;
                pairs(from, min(to, end), std::false_type{});
                vpower = all_v;
            }
            pairs(min(to, end), end, std::true_type{});
        };
        walk(keys0, keys1, values0, values1);
        bad = __syncthreads_or(bad);

        float gs = halves_sum(g);
        if (bad && (seq.cut || sees_bad_page(a, table, sp, begin, end, pos))) gs = __builtin_nanf("");
        const size_t o = (size_t)(seq.t0 + t) * a.Hq + q_head;
        if (row < rows) {
            const int v = vpower > -1000 ? vpower : 0;
            const float inv = 1.0f / gs;
            if (plan.splits > 1 && hh == 0)
                part[(size_t)a.T * a.Hq * plan.splits * D + o * plan.splits + split] = __builtin_ldexpf(gs, e);
#pragma unroll
            for (int n = 0; n < 4 * DT; ++n) {
                float f[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) f[j] = acc[n / 4][n % 4 * 4 + j];
                const int ch = 32 * (n / 4) + 8 * (n % 4) + 4 * hh;
                if (plan.splits > 1) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = __builtin_ldexpf(f[j], e + v);
                    *(float4 *)(part + (o * plan.splits + split) * D + ch) = make_float4(f[0], f[1], f[2], f[3]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        f[j] = pos < 0 ? 0.f : __builtin_ldexpf(f[j] * inv, v);   // pos < 0: sees no key
                    T *out = (T *)a.out + o * D + ch;
                    if constexpr (sizeof(T) == 2) *(uint2 *)out = make_uint2(rows::pack2(f[0], f[1]), rows::pack2(f[2], f[3]));
                    else *(float4 *)out = make_float4(f[0], f[1], f[2], f[3]);
                }
            }
        }
        __syncthreads();   // the buffers are read: another row tile may fill them
    }
}

template <typename T, int D> hipError_t launch_many(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    // Row tiles that share their keys stay on one XCD unless that leaves XCDs idle
    // or uneven (the measurements of fm_paged_chunk.hip).
    const long long units = (long long)a.S * a.Hkv * plan.splits;
    const auto more = [&](long long n) { return 7 * ((n + 7) / 8) > n || (a.S > 1 && n < 64); };
    int pieces = 1;
    while (pieces < 8 && 2 * pieces <= plan.tiles && more(units * pieces)) pieces *= 2;
    const long long blocks = (units * pieces + 7) / 8 * 8 * ((plan.tiles + pieces - 1) / pieces);
    if (!grid_fits(blocks, THREADS)) return hipErrorInvalidConfiguration;
    many_kernel<T, D><<<(unsigned)blocks, THREADS, 0, st>>>(a, plan, pieces, part);
    return hipGetLastError();
}

template <typename T, int D> hipError_t launch(const PagedArgs &a, const PagedPlan &plan, float *part, hipStream_t st)
{
    if (plan.chunk_kernel) {
        if constexpr (D >= 32) return launch_many<T, D>(a, plan, part, st);
    } else if (plan.waves == 8) {
        return launch_few<T, D, 1, 8>(a, plan, part, st);
    } else if (plan.rows == 16) {
        return launch_few<T, D, 1>(a, plan, part, st);
    } else if (plan.rows == 32) {
        return launch_few<T, D, 2>(a, plan, part, st);
    } else if constexpr (D <= 64) {
        return launch_few<T, D, 4>(a, plan, part, st);
    }
    return hipErrorInvalidValue;   // no plan has such rows
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

// The plan is the one of a bf16 cache, whatever the type of q: none of its own has been
// fitted.  Where chunks change kernels, us of the few rows' against many_kernel, 8 sequences
// of 4096 keys, 8 key heads of 4 query heads, in graphs:
//              32 rows            64 rows            128 rows
//   bf16   32  15 29              22 29              32 31
//          64  19 31              27 32              38 35
//         128  26 43              33 45              59 50
//   f32    32  16 30              24 31              37 34
//          64  21 36              41 37              62 43
//         128  37 67              51 70              94 80
// so that many_kernel, which takes over past 32 rows at D = 64 and 128 and past 64 at
// D = 32, comes too early at 64 rows: bf16 5 us at D = 64 and 12 at D = 128, float32 19 at
// D = 128.
PagedPlan paged_q8_plan(int S, int Hq, int Hkv, int D, int max_q, int max_len, int window, int sinks)
{
    return paged_plan(S, Hq, Hkv, D, 1, max_q, max_len, window, sinks, D == 128 ? 32 : 64);
}

hipError_t paged_q8_fwd(const PagedArgs &a, const PagedPlan &plan, int D, int is_bf16, void *ws, hipStream_t st)
{
    const hipError_t e = is_bf16 ? launch_d<bf16_t>(a, plan, D, (float *)ws, st) : launch_d<float>(a, plan, D, (float *)ws, st);
    return e != hipSuccess || plan.splits == 1 ? e : paged_join(a, plan, D, is_bf16, (const float *)ws, st);
}

}  // namespace fm
