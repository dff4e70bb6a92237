// Packed attention, forward (see fm_packed.h): O_i = sum_n w_in v_n / G_i,
// G_i = sum_n w_in, w_in = f_p(tau q^_i.k^_n) over the keys of the row's sequence
// (n <= i when causal).
//
// Two launches: the prep kernel standardises the keys (once for the query heads
// that share them) and scales the values; then a workgroup takes 128 rows of a
// (sequence, key head), standardises them on the way in and walks over the keys.
//
// Bound by the matrix pipe and, beside it, the weights (two fused products, half a
// conversion, half a sum and half a scale per pair): 8 prompts of up to 8192 tokens, 32
// heads to 8 of 128, bf16, 1.36 ms, 820 TFLOP/s (without loads and barriers 910 to 1075;
// a large library product reaches 1120); 16 sequences of up to 4096, 12 heads of 64, 197 us,
// 550; float32, whose MFMA rate is 153 TFLOP/s, 120 at D = 128 (2 sequences of 4096, 32
// heads to 8).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fm_internal.h"
#include "fm_packed.h"

namespace fm {
namespace packed {

// The places in the order that workgroups take them: the ones with the most work
// first, so that none is left for the end alone (16 sequences of up to 4096 tokens,
// 12 heads of 64: the last ones of each sequence at any time).  One workgroup counts
// and sorts up to SORTED of them by their tiles; more of them stay in order, many
// to every workgroup's turn.
constexpr int SORTED = 4096, BINS = 512;

template <bool BWD> __device__ __forceinline__ void plan(const PackedArgs &a, Place *out, int n, int sorted, int split, int COLS)
{
    // places of rows; then (backward) of keys, once or for dk and for dv
    const int rows = (int)((long long)a.T * a.group / COLS + a.S), keys = (int)((long long)a.T / COLS + a.S);
    // its place, and its work: tiles of the other side times the products of a tile
    const auto get = [&](int i, int &work) {
        const int role = i < rows ? ROWS : !split ? KEYS : i < rows + keys ? DK : DV;
        Place p = place_of(a.starts, a.S, a.T, role == ROWS ? a.group : 1, COLS, role == ROWS ? i : (i - rows) % keys);
        p.role = role;
        const long long other = role != ROWS ? ((long long)p.len - (a.causal ? p.first : 0)) * a.group
                                : a.causal ? min((p.first + COLS - 1) / a.group + 1, p.len) : p.len;
        const int cost = !BWD || role == KEYS ? 4 : role == DV ? 2 : 3;
        work = p.len ? (int)min((other + 63) / 64 * cost / 4, (long long)BINS - 2) + 1 : 0;
        return p;
    };
    if (!sorted) {
        const int i = blockIdx.x * THREADS + threadIdx.x;
        int work;
        if (i < n) out[n - 1 - i] = get(i, work);
        return;
    }
    __shared__ int count[BINS];
    for (int i = threadIdx.x; i < BINS; i += THREADS) count[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
        int work;
        get(i, work);
        atomicAdd(&count[BINS - 1 - work], 1);
    }
    __syncthreads();
    if (threadIdx.x < 64) {   // where each begins: 8 bins to a lane
        int sum = 0, mine[BINS / 64];
#pragma unroll
        for (int j = 0; j < BINS / 64; ++j) {
            mine[j] = sum;
            sum += count[BINS / 64 * threadIdx.x + j];
        }
        int before = sum;
        for (int o = 1; o < 64; o *= 2) {
            const int x = __shfl_up(before, o);
            if ((int)threadIdx.x >= o) before += x;
        }
#pragma unroll
        for (int j = 0; j < BINS / 64; ++j) count[BINS / 64 * threadIdx.x + j] = before - sum + mine[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS) {
        int work;
        const Place p = get(i, work);
        out[atomicAdd(&count[BINS - 1 - work], 1)] = p;
    }
}

// Blocks [0, plan_blocks): the places.  The others, one thread per 8 channels of a
// row: keys and values, then (backward) queries, dO and O.
template <typename T, int D, bool BWD>
__global__ __launch_bounds__(THREADS) void prep_kernel(PackedArgs a, Planes<typename plane_of<T>::type> p,
                                                       unsigned plan_blocks, unsigned kv_blocks)
{
    if (blockIdx.x < plan_blocks) {
        plan<BWD>(a, p.places, p.n_places, p.sorted, p.split, p.cols);
        return;
    }
    const unsigned block = blockIdx.x - plan_blocks;
    typedef typename plane_of<T>::type E;
    constexpr int L = D / 8;
    constexpr bool H = sizeof(E) == 2;
    const bool keys = !BWD || block < kv_blocks;
    const long long lane = (long long)(keys ? block : block - kv_blocks) * THREADS + threadIdx.x;
    const int c = (int)(lane % L), heads = keys ? a.Hkv : a.Hq;
    const bool ok = lane / L < (long long)a.T * heads;
    const int row = ok ? (int)(lane / L) : 0, t = row / heads, h = row - t * heads;

    const auto store = [&](E *to, const float (&x)[8]) {
        if constexpr (H) {
            h8 hi, lo;
            pr::split8<false>(x, hi, lo);
            if (ok) *(h8 *)to = hi;
        } else if (ok) {
            *(float4 *)to = make_float4(x[0], x[1], x[2], x[3]);
            *(float4 *)(to + 4) = make_float4(x[4], x[5], x[6], x[7]);
        }
    };
    const auto finite = [](float x) { return fabsf(x) <= 3.4028235e38f; };
    // x^ into a plane, 1 / std; backward: zeros for what is not finite
    const auto standard = [&](const T *from, E *to) {
        m32::RawRow<T, 8> raw;
        raw.load(from + 8 * c, ok);
        const float2 st = pr::row_stats<T, D>(raw);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = (raw.get(i) - st.x) * st.y;
            if (BWD && !finite(x[i])) x[i] = 0.f;
        }
        store(to + 8 * c, x);
        return st.y;
    };
    // a row times 2^-e, e its power, of its largest finite magnitude; returns 2 e, + 1
    // if it has what is not finite, which is left or (clean) becomes 0
    const auto scaled = [&](const m32::RawRow<T, 8> &raw, E *to, bool clean) {
        float x[8], m = 0.f, odd = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = raw.get(i);
            if (finite(x[i])) {
                m = fmaxf(m, fabsf(x[i]));
            } else {
                odd = 1.f;
                if (clean) x[i] = 0.f;
            }
        }
        int e = 0;
        if constexpr (H) {
            e = pr::exp_above(pr::group_max<L>(m));   // NO_EXP: none
            const int shift = e == pr::NO_EXP ? 0 : -e;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_ldexpf(x[i], shift);
        }
        store(to + 8 * c, x);
        return 2 * e + (pr::group_max<L>(odd) > 0.f);
    };

    if (keys) {
        const size_t at = (size_t)h * a.T + t;
        const float r = standard((const T *)a.k + t * a.ks.token + h * a.ks.head, p.kh + at * D);
        m32::RawRow<T, 8> rv;
        rv.load((const T *)a.v + t * a.vs.token + h * a.vs.head + 8 * c, ok);
        const int e = scaled(rv, p.vh + at * D, !BWD);   // backward: not contracted
        if (ok && c == 0) {
            p.b[at] = e;
            if constexpr (BWD) p.rk[at] = r;
        }
    } else if constexpr (BWD) {
        const int hk = h / a.group;
        const size_t at = ((size_t)hk * a.T + t) * a.group + (h - hk * a.group), io = (size_t)row * D + 8 * c;
        const float r = standard((const T *)a.q + t * a.qs.token + h * a.qs.head, p.qh + at * D);
        m32::RawRow<T, 8> ro, rd;
        ro.load((const T *)a.out + io, ok);
        rd.load((const T *)a.dout + io, ok);
        const int e = scaled(rd, p.oh + at * D, true), shift = e >> 1 == NO_POWER ? 0 : e >> 1;
        float delta = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            delta = fmaf(__builtin_ldexpf(rd.get(i), -shift), H ? __builtin_ldexpf(ro.get(i), -ROOM) : ro.get(i), delta);
        delta = pr::group_sum<L>(delta);
        if (ok && c == 0) {
            const float u = 1.0f / a.g[row];
            // (a row of zeros, or one whose G is not finite, has no power: it takes none
            // of the others' bits)
            RowInfo x{u, NO_POWER, delta, e & 1};
            if constexpr (H) {
                const int eu = pr::exp_above(fabsf(u));
                if (eu != pr::NO_EXP) {
                    x.m = __builtin_ldexpf(u, -eu);
                    if (e >> 1 != NO_POWER) x.e = eu + shift;
                }
                const int d = pr::exp_above(fabsf(delta));
                x.ed = 2 * (d == pr::NO_EXP ? NO_POWER : d + ROOM) + (e & 1);
            }
            p.info[at] = x;
            p.rq[at] = r;
        }
    }
}

static size_t up(size_t n) { return (n + 255) / 256 * 256; }

// 32 columns where 128 leave CUs idle (places of rows, backward of keys, times key
// heads; forward and backward in us with 32 and with 128): 12 heads of 64, 84 places
// 19 against 22 and 30 against 35, 204 26 against 33 and the same, 372 the same and 73
// against 58; 4 heads of 32, 260 53 against 86 and 140 against 166; one key head of 64
// for 8, 65 places of keys 626 against 1402; float32 4 heads of 32, 124 40 against 84
// and 80 against 161, 12 of 64, 432 310 against 355 and 912 against 855.  At D = 128 the
// tiles fill a CU's LDS: 8 heads for 32, 104 26 against 21; 12 for 12, 84 28 against 29;
// backward, places of keys, one head for 8, 33 439 against 907; 8 for 32, 56 90 against
// 117; 4 for 4, 68 69 against 80; 12 for 12, 84 64 against 48; 8 for 32, 136 320 against 280.
bool small_call(int S, int T, int Hq, int Hkv, int D, int is_bf16, int backward)
{
    if (D == 128 && !is_bf16) return false;   // LDS
    if (backward) return places(S, T, 1, 128) * Hkv < (D == 128 ? 80 : 320);
    return places(S, T, Hq / Hkv, 128) * Hkv < (D == 128 ? 96 : 448);
}

// The planes from ws on (ws null: how many bytes).
template <typename E> static Planes<E> lay_out(char *ws, int S, int T, int Hq, int Hkv, int D, int backward, size_t *bytes)
{
    size_t at = 0;
    const auto take = [&](size_t n) {
        char *const x = (char *)((uintptr_t)ws + at);
        at += up(n);
        return x;
    };
    const size_t keys = (size_t)Hkv * T, rows = (size_t)Hq * T;
    Planes<E> p = {};
    p.cols = small_call(S, T, Hq, Hkv, D, sizeof(E) == 2, backward) ? 32 : 128;
    p.split = p.cols == 128 && split_keys(D, sizeof(E) == 2);
    p.n_places = (int)(places(S, T, Hq / Hkv, p.cols) + (backward ? (p.split ? 2 : 1) * places(S, T, 1, p.cols) : 0));
    p.sorted = p.n_places <= SORTED;
    p.kh = (E *)take(keys * D * sizeof(E));
    p.vh = (E *)take(keys * D * sizeof(E));
    p.b = (int *)take(keys * sizeof(int));
    p.places = (Place *)take(p.n_places * sizeof(Place));
    if (backward) {
        p.qh = (E *)take(rows * D * sizeof(E));
        p.oh = (E *)take(rows * D * sizeof(E));
        p.rk = (float *)take(keys * sizeof(float));
        p.rq = (float *)take(rows * sizeof(float));
        p.info = (RowInfo *)take(rows * sizeof(RowInfo));
    }
    *bytes = at;
    return p;
}

template <typename E> Planes<E> planes_at(void *ws, const PackedArgs &a, int D, int backward)
{
    size_t n;
    return lay_out<E>((char *)ws, a.S, a.T, a.Hq, a.Hkv, D, backward, &n);
}
template Planes<float> planes_at(void *, const PackedArgs &, int, int);
template Planes<_Float16> planes_at(void *, const PackedArgs &, int, int);

template <typename T, int D, bool BWD>
static hipError_t prep_d(const PackedArgs &a, const Planes<typename plane_of<T>::type> &p, hipStream_t st)
{
    const long long kv = ((long long)a.T * a.Hkv * (D / 8) + THREADS - 1) / THREADS;
    const long long q = BWD ? ((long long)a.T * a.Hq * (D / 8) + THREADS - 1) / THREADS : 0;
    const long long plan = p.sorted ? 1 : (p.n_places + THREADS - 1) / THREADS;
    if (!grid_fits(plan + kv + q, THREADS)) return hipErrorInvalidConfiguration;
    prep_kernel<T, D, BWD><<<(unsigned)(plan + kv + q), THREADS, 0, st>>>(a, p, (unsigned)plan, (unsigned)kv);
    return hipGetLastError();
}

template <typename T, typename E>
hipError_t prep(const PackedArgs &a, const Planes<E> &p, int D, int backward, hipStream_t st)
{
    switch (D) {
    case 16: return backward ? prep_d<T, 16, true>(a, p, st) : prep_d<T, 16, false>(a, p, st);
    case 32: return backward ? prep_d<T, 32, true>(a, p, st) : prep_d<T, 32, false>(a, p, st);
    case 64: return backward ? prep_d<T, 64, true>(a, p, st) : prep_d<T, 64, false>(a, p, st);
    default: return backward ? prep_d<T, 128, true>(a, p, st) : prep_d<T, 128, false>(a, p, st);
    }
}
template hipError_t prep<float, float>(const PackedArgs &, const Planes<float> &, int, int, hipStream_t);
template hipError_t prep<bf16_t, _Float16>(const PackedArgs &, const Planes<_Float16> &, int, int, hipStream_t);

template <typename T, int D, int P, int WK>
__global__ __launch_bounds__(THREADS, WK == 1 ? 2 : 1) void fwd_kernel(PackedArgs a, Planes<typename plane_of<T>::type> p)
{
    typedef typename plane_of<T>::type E;
    using O = Ops<E, D>;
    using W = Cut<E, D, WK>;
    constexpr int DT = O::DT, TILE = W::TILE, MINE = W::MINE, COLS = W::COLS;
    __shared__ u4 x0[TILE * O::C], x1[TILE * O::C], y0[TILE * O::C], y1[TILE * O::C];
    __shared__ f4 factors[THREADS / 64][MINE / 4];   // whole tiles: halves; cut ones: the keys' powers
    __shared__ int wave_powers[THREADS / 64][64];
    __shared__ float wave_sums[THREADS / 64][64];

    // a key head's workgroups are Hkv apart, on one XCD where 8 divides Hkv
    const int head = blockIdx.x % a.Hkv;
    const Place pl = scalar(p.places[blockIdx.x / a.Hkv]);
    if (pl.len == 0) return;
    const int wave = scalar(threadIdx.x / 64), lane = threadIdx.x % 64, hh = lane / 32, c32 = lane % 32;
    const int rows = pl.len * a.group, wfirst = pl.first + (WK == 1 ? 32 * wave : 0);
    const int at = WK == 1 ? 0 : wave;   // the wave's first block of a tile
    const int row = wfirst + c32, t = min(row, rows - 1) / a.group;
    const int qhead = head * a.group + min(row, rows - 1) - t * a.group;
    const size_t io = (size_t)(pl.t0 + t) * a.Hq + qhead;

    typename O::Own own;
    {
        // channels of the lane's half of the row, standardised
        const T *q = (const T *)a.q + (pl.t0 + t) * a.qs.token + qhead * a.qs.head;
        float x[D / 2];
        m32::RawRow<T, 8> raw[D / 16];
#pragma unroll
        for (int k = 0; k < D / 16; ++k) raw[k].load(q + (sizeof(E) == 2 ? 16 * k + 8 * hh : hh * (D / 2) + 8 * k), true);
#pragma unroll
        for (int i = 0; i < D / 2; ++i) x[i] = raw[i / 8].get(i % 8);
        pr::standardise_cols<D>(x, true, 1.0f);
        if constexpr (sizeof(E) == 2) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                h8 hi, lo;
                pr::split8<false>(x + 8 * k, hi, lo);
                own.x[k] = __builtin_bit_cast(u4, hi);
            }
        } else {
#pragma unroll
            for (int i = 0; i < D / 2; ++i) own.x[i / 4][i % 4] = x[i];
        }
    }
    f16v acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f16v{};
    float g = 0.f;          // second order: of 2 w = (1 + tau s)^2 + 1
    int power = NO_POWER;   // of acc: the largest of the values that the row has seen
    float down = 1.f;       // 2^-power

    const int end = a.causal ? (min(pl.first + COLS, rows) - 1) / a.group + 1 : pl.len;   // keys that some row sees
    // keys before `whole` are seen by all rows, from `none` on by none of the wave's
    const int whole = (a.causal ? pl.first / a.group + 1 : pl.len) / (2 * TILE) * (2 * TILE);
    const int none = a.causal ? scalar(min(wfirst + 31, rows - 1) / a.group) + 1 : pl.len;
    const int lim = a.causal ? t : pl.len - 1;
    const size_t keys = (size_t)head * a.T + pl.t0;
    const float tau = a.tau;
    int next = p.b[keys + min(32 * at + lane % MINE, pl.len - 1)];   // the next tile's powers and marks, a key to a lane
    uint64_t odd = 0;

    // what becomes of the scores of a block of 32 keys; masked: some row does not see
    // some of them
    const auto block = [&](const f16v &s, const u4 *vt, int n1, int kb, auto masked) {
        typename O::Turned v;
        O::turn(v, vt, at + kb, lane);
        float w[16];
        const int left = lim - n1 - 4 * hh;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            w[i] = fmaf(s[i], tau, 1.0f);
            if constexpr (P == 2) w[i] = fmaf(w[i], w[i], 1.0f);
            if constexpr (decltype(masked)::value) w[i] = 8 * (i / 4) + i % 4 <= left ? w[i] : 0.f;
        }
        if constexpr (O::POWERS) {
            // the sum of the rounded weights, as the numerator takes them
            const pr::h2 one = {(_Float16)1.0f, (_Float16)1.0f};
            pr::h2 h[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                pr::h2 f[2];
                if constexpr (decltype(masked)::value) {
                    // 2^b 2^-power a row: one factor for all of them times one of the row's own
                    // would leave float32's range between a row's values and an unseen key's
                    const i4 b = ((const i4 *)factors[wave])[8 * kb + 2 * j + hh];
                    float x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = 8 * j + i <= left ? __builtin_ldexpf(down, b[i]) : 0.f;
                    f[0] = pr::cvt2(x[0], x[1]);
                    f[1] = pr::cvt2(x[2], x[3]);
                } else {
                    const h4 x = ((const h4 *)factors[wave])[8 * kb + 2 * j + hh];
                    f[0] = pr::h2{x[0], x[1]};
                    f[1] = pr::h2{x[2], x[3]};
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const pr::h2 x = pr::cvt2(w[4 * j + 2 * i], w[4 * j + 2 * i + 1]);
                    g = __builtin_amdgcn_fdot2(x, one, g, false);
                    h[2 * j + i] = x * f[i];
                }
            }
            O::add(acc, v, h);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) g += w[i];
            O::add(acc, v, w);
        }
    };
    const auto powers = [&](int n0, auto masked) {
        const int b = next >> 1;
        odd |= __ballot(next & 1);
        next = p.b[keys + min(n0 + TILE + 32 * at + lane % MINE, pl.len - 1)];
        if constexpr (O::POWERS) {
            const auto raise = [&](int most) {
                most = max(most, power);
                const float f = __builtin_ldexpf(1.0f, max(power - most, -300));
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[d] *= f;
                power = most;
            };
            if constexpr (decltype(masked)::value) {
                if (__any(wave_max(b) > power)) raise(max_to<MINE>(b, lane, lim - n0 - 32 * at));
                down = power > NO_POWER ? __builtin_ldexpf(1.0f, -power) : 1.f;
                ((int *)factors[wave])[lane % MINE] = b;
            } else {
                if (__any(b > power)) raise(wave_max(b));
                ((_Float16 *)factors[wave])[lane % MINE] = (_Float16)__builtin_ldexpf(1.0f, b - power);
            }
        }
    };
    walk<E, D, TILE>(p.kh + keys * D, p.vh + keys * D, 0, 0, whole, end, pl.len - 1, x0, x1, y0, y1, wave, lane,
                     [&](const u4 *kt, const u4 *vt, int n0) {
        powers(n0, std::false_type{});
        f16v s[MINE / 32];
#pragma unroll
        for (int kb = 0; kb < MINE / 32; ++kb) s[kb] = O::scores(kt, at + kb, hh, c32, own);
#pragma unroll
        for (int kb = 0; kb < MINE / 32; ++kb) block(s[kb], vt, n0 + 32 * (at + kb), kb, std::false_type{});
    },
                     [&](const u4 *kt, const u4 *vt, int n0) {
        powers(n0, std::true_type{});
#pragma unroll
        for (int kb = 0; kb < MINE / 32; ++kb)
            if (n0 + 32 * (at + kb) < none)
                block(O::scores(kt, at + kb, hh, c32, own), vt, n0 + 32 * (at + kb), kb, std::true_type{});
    });
    if constexpr (WK > 1) {
        u4 *const mine = wave == 0 ? x0 : wave == 1 ? x1 : wave == 2 ? y0 : y1;   // free: the last tile is behind a barrier
        wave_sums[wave][lane] = g;
        join_put<DT>(acc, power, wave_powers, mine, wave, lane);
        odd = __syncthreads_or(odd != 0);
        if (wave) return;
        join_get<DT>(acc, x0, x1, y0, y1, lane);
        g = (wave_sums[0][lane] + wave_sums[1][lane]) + (wave_sums[2][lane] + wave_sums[3][lane]);
    }

    const float G = pr::half_sum(g);
    // out of the power in two factors: each a normal number
    const float f = 1.0f / G;
    const int e0 = O::POWERS && power > NO_POWER ? power / 2 : 0, e1 = O::POWERS && power > NO_POWER ? power - e0 : 0;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = __builtin_ldexpf(__builtin_ldexpf(acc[d][i], e0) * f, e1);
    if (odd)
        add_odd<T, D>(acc, 0, none, lane, [&](int n) { return p.b[keys + n] & 1; },
                      [&](int n) { return (const T *)a.v + (pl.t0 + n) * a.vs.token + head * a.vs.head; },
                      [&](int n) { return n <= lim; });
    if (row >= rows) return;
    if (a.g && hh == 0) a.g[io] = P == 2 ? 0.5f * G : G;
    store_row<T, D>((T *)a.out + io * D, acc, hh);
}

template <typename T, int D> hipError_t launch(const PackedArgs &a, void *ws, hipStream_t st)
{
    typedef typename plane_of<T>::type E;
    const Planes<E> p = planes_at<E>(ws, a, D, 0);
    const long long blocks = (long long)p.n_places * a.Hkv;
    if (!grid_fits(blocks, THREADS)) return hipErrorInvalidConfiguration;
    const hipError_t e = prep<T, E>(a, p, D, 0, st);
    if (e != hipSuccess) return e;
    if constexpr (Cut<E, D, 4>::FITS) {
        if (p.cols == 32) {
            if (a.p == 2) fwd_kernel<T, D, 2, 4><<<(unsigned)blocks, THREADS, 0, st>>>(a, p);
            else fwd_kernel<T, D, 1, 4><<<(unsigned)blocks, THREADS, 0, st>>>(a, p);
            return hipGetLastError();
        }
    }
    if (a.p == 2) fwd_kernel<T, D, 2, 1><<<(unsigned)blocks, THREADS, 0, st>>>(a, p);
    else fwd_kernel<T, D, 1, 1><<<(unsigned)blocks, THREADS, 0, st>>>(a, p);
    return hipGetLastError();
}

template <typename T> hipError_t launch_d(const PackedArgs &a, int D, void *ws, hipStream_t st)
{
    switch (D) {
    case 16: return launch<T, 16>(a, ws, st);
    case 32: return launch<T, 32>(a, ws, st);
    case 64: return launch<T, 64>(a, ws, st);
    default: return launch<T, 128>(a, ws, st);
    }
}

}  // namespace packed

size_t packed_workspace(int S, int T, int Hq, int Hkv, int D, int is_bf16, int backward)
{
    size_t n;
    if (is_bf16) packed::lay_out<_Float16>(nullptr, S, T, Hq, Hkv, D, backward, &n);
    else packed::lay_out<float>(nullptr, S, T, Hq, Hkv, D, backward, &n);
    return n;
}

hipError_t packed_fwd(const PackedArgs &a, int D, int is_bf16, void *ws, hipStream_t st)
{
    return is_bf16 ? packed::launch_d<bf16_t>(a, D, ws, st) : packed::launch_d<float>(a, D, ws, st);
}

}  // namespace fm
