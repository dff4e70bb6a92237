// Packed attention, forward (see fm_packed.h): O_i = sum_n w_in v_n / G_i,
// G_i = sum_n w_in, w_in = f_p(tau q^_i.k^_n) over the keys of the row's sequence
// (n <= i when causal).
//
// Two launches: the prep kernel standardises the keys (once for the query heads
// that share them) and scales the values; then a workgroup takes 128 rows of a
// (sequence, key head), standardises them on the way in and walks over the keys.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fm_internal.h"
#include "fm_packed.h"

namespace fm {
namespace packed {

// One thread per 8 channels of a row; blocks [0, kv_blocks): keys and values, the
// others (backward): queries, dO and O.
template <typename T, int D, bool BWD>
__global__ __launch_bounds__(THREADS) void prep_kernel(PackedArgs a, Planes<typename plane_of<T>::type> p, unsigned kv_blocks)
{
    typedef typename plane_of<T>::type E;
    constexpr int L = D / 8;
    constexpr bool H = sizeof(E) == 2;
    const bool keys = !BWD || blockIdx.x < kv_blocks;
    const long long lane = (long long)(keys ? blockIdx.x : blockIdx.x - kv_blocks) * THREADS + threadIdx.x;
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
    // x^ into a plane, 1 / std
    const auto standard = [&](const T *from, E *to) {
        m32::RawRow<T, 8> raw;
        raw.load(from + 8 * c, ok);
        const float2 st = pr::row_stats<T, D>(raw);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (raw.get(i) - st.x) * st.y;
        store(to + 8 * c, x);
        return st.y;
    };
    // a row times 2^-e, e its power (returned): of its largest finite magnitude
    const auto scaled = [&](const m32::RawRow<T, 8> &raw, E *to) {
        float x[8], m = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = raw.get(i);
            m = fmaxf(m, fabsf(x[i]) <= 3.4028235e38f ? fabsf(x[i]) : 0.f);
        }
        int e = NO_POWER;
        if constexpr (H) {
            e = pr::exp_above(pr::group_max<L>(m));   // NO_EXP: none
            const int shift = e == pr::NO_EXP ? 0 : -e;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_ldexpf(x[i], shift);
        }
        store(to + 8 * c, x);
        return e;
    };

    if (keys) {
        const size_t at = (size_t)h * a.T + t;
        const float r = standard((const T *)a.k + t * a.ks.token + h * a.ks.head, p.kh + at * D);
        m32::RawRow<T, 8> rv;
        rv.load((const T *)a.v + t * a.vs.token + h * a.vs.head + 8 * c, ok);
        const int e = scaled(rv, p.vh + at * D);
        if (ok && c == 0) {
            if constexpr (H) p.b[at] = e;
            if constexpr (BWD) p.rk[at] = r;
        }
    } else if constexpr (BWD) {
        const int hk = h / a.group;
        const size_t at = ((size_t)hk * a.T + t) * a.group + (h - hk * a.group), io = (size_t)row * D + 8 * c;
        const float r = standard((const T *)a.q + t * a.qs.token + h * a.qs.head, p.qh + at * D);
        m32::RawRow<T, 8> ro, rd;
        ro.load((const T *)a.out + io, ok);
        rd.load((const T *)a.dout + io, ok);
        const int e = scaled(rd, p.oh + at * D), shift = H && e != NO_POWER ? e : 0;
        float delta = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) delta = fmaf(__builtin_ldexpf(rd.get(i), -shift), ro.get(i), delta);
        delta = pr::group_sum<L>(delta);
        if (ok && c == 0) {
            const float u = 1.0f / a.g[row];
            RowInfo x{u, 0, delta, 0};
            if constexpr (H) {
                const int eu = pr::exp_above(fabsf(u));
                if (eu != pr::NO_EXP) {
                    x.m = __builtin_ldexpf(u, -eu);
                    x.e = eu + shift;
                }
                x.ed = pr::exp_above(fabsf(delta));
            }
            p.info[at] = x;
            p.rq[at] = r;
        }
    }
}

static size_t up(size_t n) { return (n + 255) / 256 * 256; }

template <typename E> Planes<E> planes_at(void *ws, int T, int Hq, int Hkv, int D, int backward)
{
    char *at = (char *)ws;
    const auto take = [&](size_t n) {
        char *const x = at;
        at += up(n);
        return x;
    };
    const size_t keys = (size_t)Hkv * T, rows = (size_t)Hq * T;
    Planes<E> p = {};
    p.kh = (E *)take(keys * D * sizeof(E));
    p.vh = (E *)take(keys * D * sizeof(E));
    p.b = (int *)take(sizeof(E) == 2 ? keys * sizeof(int) : 0);
    if (backward) {
        p.qh = (E *)take(rows * D * sizeof(E));
        p.oh = (E *)take(rows * D * sizeof(E));
        p.rk = (float *)take(keys * sizeof(float));
        p.rq = (float *)take(rows * sizeof(float));
        p.info = (RowInfo *)take(rows * sizeof(RowInfo));
    }
    return p;
}
template Planes<float> planes_at(void *, int, int, int, int, int);
template Planes<_Float16> planes_at(void *, int, int, int, int, int);

size_t planes_bytes(int T, int Hq, int Hkv, int D, int is_bf16, int backward)
{
    const size_t keys = (size_t)Hkv * T, rows = (size_t)Hq * T, e = is_bf16 ? 2 : 4;
    size_t n = 2 * up(keys * D * e) + (is_bf16 ? up(keys * sizeof(int)) : 0);
    if (backward)
        n += 2 * up(rows * D * e) + up(keys * sizeof(float)) + up(rows * sizeof(float)) + up(rows * sizeof(RowInfo));
    return n;
}

template <typename T, int D, bool BWD>
static hipError_t prep_d(const PackedArgs &a, const Planes<typename plane_of<T>::type> &p, hipStream_t st)
{
    const long long kv = ((long long)a.T * a.Hkv * (D / 8) + THREADS - 1) / THREADS;
    const long long q = BWD ? ((long long)a.T * a.Hq * (D / 8) + THREADS - 1) / THREADS : 0;
    if (!grid_fits(kv + q, THREADS)) return hipErrorInvalidConfiguration;
    prep_kernel<T, D, BWD><<<(unsigned)(kv + q), THREADS, 0, st>>>(a, p, (unsigned)kv);
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

template <typename T, int D, int P>
__global__ __launch_bounds__(THREADS, 2) void fwd_kernel(PackedArgs a, Planes<typename plane_of<T>::type> p, int groups)
{
    typedef typename plane_of<T>::type E;
    using O = Ops<E, D>;
    constexpr int DT = O::DT, TILE = O::TILE;
    __shared__ u4 x0[TILE * O::C], x1[TILE * O::C], y0[TILE * O::C], y1[TILE * O::C];
    __shared__ f4 factors[THREADS / 64][TILE / 4];

    // the last rows see the most keys and start first; a key head's workgroups
    // are Hkv apart, on one XCD where 8 divides Hkv
    const int head = blockIdx.x % a.Hkv;
    const Place pl = place_of(a.starts, a.S, a.T, a.group, groups - 1 - blockIdx.x / a.Hkv);
    if (pl.len == 0) return;
    const int wave = scalar(threadIdx.x / 64), lane = threadIdx.x % 64, hh = lane / 32, c32 = lane % 32;
    const int rows = pl.len * a.group, wfirst = pl.first + 32 * wave;
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
    float g = 0.f;
    int power = NO_POWER;   // of acc: the largest of the values' so far

    const int end = a.causal ? (min(pl.first + COLS, rows) - 1) / a.group + 1 : pl.len;   // keys that some row sees
    // the wave's: keys before `whole` are seen by all its rows, from `none` on by none
    const int whole = a.causal ? scalar(min(wfirst, rows - 1) / a.group) + 1 : pl.len;
    const int none = a.causal ? scalar(min(wfirst + 31, rows - 1) / a.group) + 1 : pl.len;
    const int lim = a.causal ? t : pl.len - 1;
    const size_t keys = (size_t)head * a.T + pl.t0;
    const float c1 = a.tau, c2 = 0.5f * a.tau * a.tau;
    int next = 0;   // the next tile's powers, a key to a lane
    if constexpr (O::POWERS) next = p.b[keys + min(lane, pl.len - 1)];

    walk<E, D>(p.kh + keys * D, p.vh + keys * D, 0, end, pl.len - 1, x0, x1, y0, y1, wave, lane,
               [&](const u4 *kt, const u4 *vt, int n0) {
        if constexpr (O::POWERS) {
            const int b = next;
            next = p.b[keys + min(n0 + TILE + lane, pl.len - 1)];
            const int most = wave_max(b);
            if (most > power) {
                const float f = __builtin_ldexpf(1.0f, max(power - most, -300));
#pragma unroll
                for (int d = 0; d < DT; ++d) acc[d] *= f;
                power = most;
            }
            ((float *)factors[wave])[lane] = __builtin_ldexpf(1.0f, b - power);
        }
#pragma unroll
        for (int kb = 0; kb < TILE / 32; ++kb) {
            const int n1 = n0 + 32 * kb;
            if (n1 >= none) break;
            f16v s = O::scores(kt, kb, hh, c32, own);
            typename O::Turned v;
            O::turn(v, vt, kb, lane);
            float w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = P == 2 ? fmaf(fmaf(s[i], c2, c1), s[i], 1.0f) : fmaf(s[i], c1, 1.0f);
            uint32_t seen = 0xffffu;
            const bool all = n1 + 32 <= whole;
            if (!all) {
                seen = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool see = n1 + 8 * (i / 4) + 4 * hh + i % 4 <= lim;
                    w[i] = see ? w[i] : 0.f;
                    seen |= (uint32_t)see << i;
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) g += w[i];
            if constexpr (O::POWERS) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f4 f = factors[wave][8 * kb + 2 * j + hh];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[4 * j + i] *= f[i];
                }
            }
            if (all) O::add(acc, v, w);
            else add_masked<E, D>(acc, vt, kb, lane, v, w, seen);
        }
    });

    const float G = pr::half_sum(g);
    if (row >= rows) return;
    if (a.g && hh == 0) a.g[io] = G;
    // out of the power in two factors: each a normal number
    const float f = 1.0f / G;
    const int e0 = O::POWERS && power > NO_POWER ? power / 2 : 0, e1 = O::POWERS && power > NO_POWER ? power - e0 : 0;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = __builtin_ldexpf(__builtin_ldexpf(acc[d][i], e0) * f, e1);
    store_row<T, D>((T *)a.out + io * D, acc, hh);
}

template <typename T, int D> hipError_t launch(const PackedArgs &a, void *ws, hipStream_t st)
{
    typedef typename plane_of<T>::type E;
    const long long groups = workgroups(a.S, a.T, a.group);
    if (!grid_fits(groups * a.Hkv, THREADS)) return hipErrorInvalidConfiguration;
    const Planes<E> p = planes_at<E>(ws, a.T, a.Hq, a.Hkv, D, 0);
    const hipError_t e = prep<T, E>(a, p, D, 0, st);
    if (e != hipSuccess) return e;
    const unsigned blocks = (unsigned)(groups * a.Hkv);
    if (a.p == 2) fwd_kernel<T, D, 2><<<blocks, THREADS, 0, st>>>(a, p, (int)groups);
    else fwd_kernel<T, D, 1><<<blocks, THREADS, 0, st>>>(a, p, (int)groups);
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

size_t packed_workspace(int T, int Hq, int Hkv, int D, int is_bf16, int backward)
{
    return packed::planes_bytes(T, Hq, Hkv, D, is_bf16, backward);
}

hipError_t packed_fwd(const PackedArgs &a, int D, int is_bf16, void *ws, hipStream_t st)
{
    return is_bf16 ? packed::launch_d<bf16_t>(a, D, ws, st) : packed::launch_d<float>(a, D, ws, st);
}

}  // namespace fm
