// Packed attention, backward (see fm_packed.h), from O and G as the other
// backwards (Sec. 2.5): with u = 1 / G, delta_i = dO_i.O_i, t = f_p'(tau s),
//   T_in  = t u_i (dO_i.v_n - delta_i)                (Sec. 2.3, Eq. "bound")
//   dq^_i = tau sum_n T_in k^_n,  dk^_n = tau sum_i T_in q^_i,
//   dv_n  = sum_i w_in u_i dO_i,
// sums over i with every query head of the group, then the standardisation
// backward, dx = (dx^ - mean dx^ - x^ mean(dx^ x^)) / std (Eqs. 6-7).
//
// The prep kernel writes q^, k^, v, dO as planes and a few words per row; one launch
// holds two kinds of workgroups: of 128 rows over the keys (dq), and of 128 keys
// over the rows (dk and dv, which share their scores).  No atomics: every output
// row has one owner, equal calls give equal bits.
//
// Seven products a pair of rows and keys (scores, dO.v and dq for the rows; scores, dO.v,
// dk and dv for the keys), eight where dk and dv have workgroups of their own (3 + 3 + 2),
// and, beside them, the weights and T, made as often as the scores; five products and one
// making would do if all sums had one owner.  16 sequences of up to 4096, 12 heads of 64,
// bf16, 615 us, 440 TFLOP/s of the five; 5 of up to 4095, 32 heads to 8 of 128, 960 us, 510;
// the prep kernel is 75 us of the first.  float32, D = 128: 86 of 153 TFLOP/s.
//
// Powers of two (bf16 calls).  With dO_i = 2^a_i o_i, v_n = 2^b_n x_n and
// delta_i = 2^a_i d_i:
//   rows:  T 2^-(a_i + E) / u_i = t (2^(b_n - E) o_i.x_n - 2^-E d_i), E >= every b_n seen so
//          far and d_i, so that t (.) stays below (1 + D)^2 < 2^15;
//   keys:  u_i 2^a_i = m_i 2^e_i, M >= every e_i seen so far, F >= b_n and every d_i seen so
//          far:  T 2^-(M + F) = t (X_i 2^(b_n - F) o_i.x_n - Y_i),  X_i = m_i 2^(e_i - M),
//          Y_i = X_i d_i 2^-F,  and w X_i for dv.
// A wave that meets a larger one scales its sums down.  E is a row's own; M and F are a
// key's own in the tiles that the mask cuts, then the wave's.  A row of zeros has no e_i.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fm_internal.h"
#include "fm_packed.h"

namespace fm {
namespace packed {

// The standardisation backward of a wave's columns in place: x^ from the plane's
// row, r = 1 / std.
template <typename E, int D>
__device__ __forceinline__ void standardise_back(const E *row, float r, f16v *acc, int hh)
{
    using O = Ops<E, D>;
    float x[O::DT][16], m1 = 0.f, m2 = 0.f;
#pragma unroll
    for (int d = 0; d < O::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int ch = O::channel(d, i, hh);
            const bool in = D >= 32 || ch < D;
            x[d][i] = in ? (float)row[in ? ch : 0] : 0.f;
            if (!in) acc[d][i] = 0.f;
            m1 += acc[d][i];
            m2 = fmaf(acc[d][i], x[d][i], m2);
        }
    m1 = pr::half_sum(m1) * (1.0f / D);
    m2 = pr::half_sum(m2) * (1.0f / D);
#pragma unroll
    for (int d = 0; d < O::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = (acc[d][i] - m1 - x[d][i] * m2) * r;
}

// acc times f 2^e, in steps that stay normal numbers.
template <int DT>
__device__ __forceinline__ void scale_up(f16v *acc, float f, int e)
{
    const int e0 = e / 2, e1 = e - e0;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = __builtin_ldexpf(__builtin_ldexpf(acc[d][i], e0) * f, e1);
}
template <int DT>
__device__ __forceinline__ void scale_down(f16v *acc, int e)
{
    const float f = __builtin_ldexpf(1.0f, max(e, -300));
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] *= f;
}

template <typename T, int D, int P, int WK>
__device__ __forceinline__ void rows_block(const PackedArgs &a, const Planes<typename plane_of<T>::type> &p, int head,
                                           const Place &pl, u4 *x0, u4 *x1, u4 *y0, u4 *y1, f4 *factors, int (*wave_powers)[64])
{
    typedef typename plane_of<T>::type E;
    using O = Ops<E, D>;
    using W = Cut<E, D, WK>;
    constexpr int DT = O::DT, TILE = W::TILE, MINE = W::MINE, COLS = W::COLS;
    const int wave = scalar(threadIdx.x / 64), lane = threadIdx.x % 64, hh = lane / 32, c32 = lane % 32;
    const int rows = pl.len * a.group, wfirst = pl.first + (WK == 1 ? 32 * wave : 0);
    const int at = WK == 1 ? 0 : wave;   // the wave's first block of a tile
    const int row = min(wfirst + c32, rows - 1), t = row / a.group;
    const size_t base = ((size_t)head * a.T + pl.t0) * a.group, keys = (size_t)head * a.T + pl.t0;

    typename O::Own q, o;
    O::own(q, p.qh + (base + row) * D, hh);
    O::own(o, p.oh + (base + row) * D, hh);
    const RowInfo info = p.info[base + row];
    f16v acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[d] = f16v{};
    int power = O::POWERS ? info.ed >> 1 : 0;   // E
    int all = NO_POWER;                         // the tiles' so far
    // whole tiles: delta 2^-R and 2^(R - E), R what the factors are relative to; cut ones:
    // delta 2^-E and 2^-E
    float delta = info.delta, up = 1.f;
    const auto relative = [&](int to) {
        // (values 2^60 below E vanish in any case)
        const int R = max(to, power - 60);
        delta = __builtin_ldexpf(info.delta, ROOM - R);
        up = __builtin_ldexpf(1.0f, min(R - power, 120));
    };
    if constexpr (O::POWERS) relative(all);

    const int end = a.causal ? (min(pl.first + COLS, rows) - 1) / a.group + 1 : pl.len;
    const int whole = (a.causal ? pl.first / a.group + 1 : pl.len) / (2 * TILE) * (2 * TILE);
    const int none = a.causal ? scalar(min(wfirst + 31, rows - 1) / a.group) + 1 : pl.len;
    const int lim = a.causal ? t : pl.len - 1;
    const float tau = a.tau;
    int next = p.b[keys + min(32 * at + lane % MINE, pl.len - 1)];

    const auto block = [&](const f16v &s, const f16v &dp, const u4 *kt, int n1, int kb, auto masked) {
        typename O::Turned k;
        O::turn(k, kt, at + kb, lane);
        float w[16];
        const int left = lim - n1 - 4 * hh;
        // (in a cut tile a row's own factors: 2^b 2^-E has no part that an unseen key's
        // power could take out of float32's range)
        constexpr bool OWN = O::POWERS && decltype(masked)::value;
        const float t1 = OWN ? 1.f : up, tau1 = OWN ? tau : tau * up;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f4 f;
            if constexpr (OWN) {
                const i4 b = ((const i4 *)factors)[8 * kb + 2 * j + hh];
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = __builtin_ldexpf(up, b[i]);
            } else if constexpr (O::POWERS) {
                f = factors[8 * kb + 2 * j + hh];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = O::POWERS ? fmaf(dp[4 * j + i], f[i], -delta) : dp[4 * j + i] - delta;
                float x = P == 2 ? fmaf(s[4 * j + i], tau1, t1) * d : O::POWERS ? t1 * d : d;
                if constexpr (decltype(masked)::value) x = 8 * j + i <= left ? x : 0.f;
                w[4 * j + i] = x;
            }
        }
        O::add(acc, k, w);
    };
    const auto powers = [&](int n0, auto masked) {
        if constexpr (O::POWERS) {
            const int b = next >> 1;
            next = p.b[keys + min(n0 + TILE + 32 * at + lane % MINE, pl.len - 1)];
            const auto raise = [&](int most) {
                most = max(most, power);
                scale_down<DT>(acc, power - most);
                power = most;
            };
            if constexpr (decltype(masked)::value) {
                if (__any(wave_max(b) > power)) raise(max_to<MINE>(b, lane, lim - n0 - 32 * at));
                up = power > NO_POWER ? __builtin_ldexpf(1.0f, -power) : 1.f;
                delta = power > NO_POWER ? __builtin_ldexpf(info.delta, ROOM - power) : info.delta;
                ((int *)factors)[lane % MINE] = b;
            } else {
                if (__any(b > all)) {
                    all = max(all, wave_max(b));
                    if (__any(all > power)) raise(all);
                    relative(all);
                }
                ((float *)factors)[lane % MINE] = __builtin_ldexpf(1.0f, b - all);
            }
        }
    };
    const auto scores = [&](const u4 *kt, const u4 *vt, int kb, f16v &s, f16v &dp) {
        O::scores2(kt, at + kb, q, s, vt, at + kb, o, dp, hh, c32);
    };
    walk<E, D, TILE>(p.kh + keys * D, p.vh + keys * D, 0, 0, whole, end, pl.len - 1, x0, x1, y0, y1, wave, lane,
                     [&](const u4 *kt, const u4 *vt, int n0) {
        powers(n0, std::false_type{});
        if constexpr (ahead<E, D>()) {
            f16v s[MINE / 32], dp[MINE / 32];
#pragma unroll
            for (int kb = 0; kb < MINE / 32; ++kb) scores(kt, vt, kb, s[kb], dp[kb]);
#pragma unroll
            for (int kb = 0; kb < MINE / 32; ++kb) block(s[kb], dp[kb], kt, n0 + 32 * (at + kb), kb, std::false_type{});
        } else {
#pragma unroll
            for (int kb = 0; kb < MINE / 32; ++kb) {
                f16v s, dp;
                scores(kt, vt, kb, s, dp);
                block(s, dp, kt, n0 + 32 * (at + kb), kb, std::false_type{});
            }
        }
    },
                     [&](const u4 *kt, const u4 *vt, int n0) {
        powers(n0, std::true_type{});
#pragma unroll
        for (int kb = 0; kb < MINE / 32; ++kb) {
            if (n0 + 32 * (at + kb) >= none) break;
            f16v s, dp;
            scores(kt, vt, kb, s, dp);
            block(s, dp, kt, n0 + 32 * (at + kb), kb, std::true_type{});
        }
    });
    if constexpr (WK > 1) {
        join_put<DT>(acc, power, wave_powers, wave == 0 ? x0 : wave == 1 ? x1 : wave == 2 ? y0 : y1, wave, lane);
        __syncthreads();
        if (wave) return;
        join_get<DT>(acc, x0, x1, y0, y1, lane);
    }

    if (O::POWERS) scale_up<DT>(acc, tau * info.m, info.e + (power > NO_POWER ? power : 0));
    else scale_up<DT>(acc, tau * info.m, 0);
    standardise_back<E, D>(p.qh + (base + row) * D, p.rq[base + row], acc, hh);
    if (wfirst + c32 >= rows) return;
    store_row<T, D>((T *)a.dq + (pl.t0 + t) * a.dqs.token + (head * a.group + row - t * a.group) * a.dqs.head, acc, hh);
}

template <typename T, int D, int P, int ROLE, int WK>
__device__ __forceinline__ void keys_block(const PackedArgs &a, const Planes<typename plane_of<T>::type> &p, int head,
                                           const Place &pl, u4 *x0, u4 *x1, u4 *y0, u4 *y1, f4 *factors, int (*wave_powers)[64])
{
    typedef typename plane_of<T>::type E;
    using O = Ops<E, D>;
    using W = Cut<E, D, WK>;
    constexpr int DT = O::DT, TILE = W::TILE, MINE = W::MINE, COLS = W::COLS;
    constexpr bool GK = ROLE != DV, GV = ROLE != DK;
    const int wave = scalar(threadIdx.x / 64), lane = threadIdx.x % 64, hh = lane / 32, c32 = lane % 32;
    const int rows = pl.len * a.group, wfirst = pl.first + (WK == 1 ? 32 * wave : 0);
    const int at = WK == 1 ? 0 : wave;   // the wave's first block of a tile
    const int n = min(wfirst + c32, pl.len - 1);
    const size_t base = ((size_t)head * a.T + pl.t0) * a.group, keys = (size_t)head * a.T + pl.t0;

    typename O::Own k, v;
    O::own(k, p.kh + (keys + n) * D, hh);
    f16v dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[d] = dv[d] = f16v{};
    int b = 0, M = NO_POWER, F = 0;   // the column's power; the largest so far
    bool shared = false;              // whether M and F are the wave's
    float cx = 1.f, cy = 1.f;         // 2^-M and 2^-F times the tile's largest
    // the column's values in the power F
    const auto own_values = [&] {
        if constexpr (GK) O::own(v, p.vh + (keys + n) * D, hh);
        if constexpr (GK && O::POWERS) {
            const _Float16 f = pr::half2i(b - F);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) v.x[i] = __builtin_bit_cast(u4, __builtin_bit_cast(h8, v.x[i]) * f);
        }
    };
    if constexpr (O::POWERS) {
        F = b = p.b[keys + n] >> 1;
    }
    own_values();

    // rows of tokens from the workgroup's (the wave's) first key on see it; all keys
    // are seen by rows of the last key's token and later
    const int begin = a.causal ? pl.first * a.group / TILE * TILE : 0;
    const int some = a.causal ? min(wfirst, pl.len - 1) * a.group : 0;
    const int whole = begin + (a.causal ? (min(pl.first + COLS - 1, pl.len - 1) * a.group - begin + 2 * TILE - 1) / (2 * TILE) * (2 * TILE) : 0);
    const int least = a.causal ? n * a.group : 0;
    const float tau = a.tau;
    RowInfo next = p.info[base + min(begin + 32 * at + lane % MINE, rows - 1)];
    uint64_t odd = 0;

    const auto block = [&](const f16v &s, const f16v &dp, const u4 *qt, const u4 *ot, int r1, int kb, auto masked) {
        float w[16], x[16];
        const int lim = least - r1 - 4 * hh;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f4 fx = factors[8 * kb + 2 * j + hh], fy = factors[16 + 8 * kb + 2 * j + hh];
            if constexpr (O::POWERS && decltype(masked)::value) {
                fx *= cx;
                fy = fy * cx * cy;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // f_1, and f_2'; 2 f_2 = t^2 + 1
                const float t = fmaf(s[4 * j + i], tau, 1.0f);
                const float d = GK ? fmaf(dp[4 * j + i], fx[i], -fy[i]) : 0.f;
                float wi = P == 2 ? fmaf(t, t, 1.0f) * fx[i] : t * fx[i], xi = P == 2 ? t * d : d;
                if constexpr (decltype(masked)::value) {
                    const bool see = 8 * j + i >= lim;
                    wi = see ? wi : 0.f;
                    xi = see ? xi : 0.f;
                }
                w[4 * j + i] = wi;
                x[4 * j + i] = xi;
            }
        }
        typename O::Turned xt;
        if constexpr (GK) {
            O::turn(xt, qt, at + kb, lane);
            O::add(dk, xt, x);
        }
        if constexpr (GV) {
            O::turn(xt, ot, at + kb, lane);
            O::add(dv, xt, w);
        }
    };
    const auto powers = [&](int r0, auto masked) {
        const RowInfo info = next;
        odd |= __ballot(info.ed & 1);
        next = p.info[base + min(r0 + TILE + 32 * at + lane % MINE, rows - 1)];
        float X = info.m, Y = info.m * info.delta;
        if constexpr (O::POWERS) {
            const auto raise = [&](int m, int f) {
                scale_down<DT>(dv, M - m);
                if constexpr (GK) scale_down<DT>(dk, M - m + F - f);
                M = m;
                if (GK && __any(f > F)) {
                    F = f;
                    own_values();
                }
            };
            if constexpr (decltype(masked)::value) {
                const int e = wave_max(info.e), d = GK ? wave_max(info.ed >> 1) : NO_POWER;
                if (__any(e > M || d > F)) {
                    const int from = least - r0 - 32 * at;
                    const int m = max(M, max_from<MINE>(info.e, lane, from));
                    const int f = GK ? max(F, max_from<MINE>(info.ed >> 1, lane, from)) : F;
                    raise(m, f);
                }
                cx = __builtin_ldexpf(1.0f, min(e - M, 126));
                cy = __builtin_ldexpf(1.0f, min(d - F, 126));
                X = __builtin_ldexpf(info.m, info.e - e);
                Y = X * __builtin_ldexpf(info.delta, ROOM - d);
            } else {
                if (!shared) {
                    // the least of the columns', which keeps all their bits (within
                    // 2^40, for what the sums have room for)
                    const int m = max(wave_min(M), wave_max(M) - 40);
                    const int f = GK ? max(wave_max(b), max(wave_min(F), wave_max(F) - 40)) : F;
#pragma unroll
                    for (int x = 0; x < DT; ++x) {
                        dv[x] *= __builtin_ldexpf(1.0f, max(M - m, -300));
                        if constexpr (GK) dk[x] *= __builtin_ldexpf(1.0f, max(M - m + F - f, -300));
                    }
                    M = m;
                    F = f;
                    own_values();
                    shared = true;
                }
                if (__any(info.e > M || (GK && info.ed >> 1 > F)))
                    raise(max(M, wave_max(info.e)), GK ? max(F, wave_max(info.ed >> 1)) : F);
                X = __builtin_ldexpf(info.m, info.e - M);
                Y = X * __builtin_ldexpf(info.delta, ROOM - F);
            }
        }
        // rows past the last weigh nothing
        if (r0 + 32 * at + lane % MINE >= rows) X = Y = 0.f;
        if (MINE == 64 || lane < 32) {
            ((float *)factors)[lane] = X;
            ((float *)(factors + 16))[lane] = Y;
        }
    };
    const auto scores = [&](const u4 *qt, const u4 *ot, int kb, f16v &s, f16v &dp) {
        if constexpr (GK) O::scores2(qt, at + kb, k, s, ot, at + kb, v, dp, hh, c32);
        else s = O::scores(qt, at + kb, hh, c32, k);
    };
    walk<E, D, TILE>(p.qh + base * D, p.oh + base * D, begin, min(whole, rows), rows, rows, rows - 1, x0, x1,
                     y0, y1, wave, lane,
                     [&](const u4 *qt, const u4 *ot, int r0) {
        powers(r0, std::false_type{});
        if constexpr (ROLE == DV || (ROLE == DK && ahead<E, D>())) {
            f16v s[MINE / 32], dp[MINE / 32];
#pragma unroll
            for (int kb = 0; kb < MINE / 32; ++kb) scores(qt, ot, kb, s[kb], dp[kb]);
#pragma unroll
            for (int kb = 0; kb < MINE / 32; ++kb) block(s[kb], dp[kb], qt, ot, r0 + 32 * (at + kb), kb, std::false_type{});
        } else {
#pragma unroll
            for (int kb = 0; kb < MINE / 32; ++kb) {
                f16v s, dp;
                scores(qt, ot, kb, s, dp);
                block(s, dp, qt, ot, r0 + 32 * (at + kb), kb, std::false_type{});
            }
        }
    },
                     [&](const u4 *qt, const u4 *ot, int r0) {
        powers(r0, std::true_type{});
#pragma unroll
        for (int kb = 0; kb < MINE / 32; ++kb) {
            const int r1 = r0 + 32 * (at + kb);
            if (r1 + 31 < some || r1 >= rows) continue;
            f16v s, dp;
            scores(qt, ot, kb, s, dp);
            block(s, dp, qt, ot, r1, kb, std::true_type{});
        }
    });
    // powers of the sums; a wave without a block of its own has none
    int ek = !O::POWERS ? 0 : M > NO_POWER ? M + (F > NO_POWER ? F : 0) : NO_POWER, ev = O::POWERS ? M : 0;
    if constexpr (WK > 1) {
        u4 *const mine = wave == 0 ? x0 : wave == 1 ? x1 : wave == 2 ? y0 : y1;
        join_put<DT>(dk, ek, wave_powers, mine, wave, lane);
        odd = __syncthreads_or(odd != 0);
        if (wave == 0) join_get<DT>(dk, x0, x1, y0, y1, lane);
        __syncthreads();
        join_put<DT>(dv, ev, wave_powers, mine, wave, lane);
        __syncthreads();
        if (wave > 1) return;
        if (wave == 1) join_get<DT>(dv, x0, x1, y0, y1, lane);
    }
    ek = ek > NO_POWER ? ek : 0;
    ev = ev > NO_POWER ? ev : 0;
    const size_t tok = pl.t0 + n;
    const bool mine = wfirst + c32 < pl.len;
    if (GK && (WK == 1 || wave == 0)) {
        scale_up<DT>(dk, a.tau, ek);
        standardise_back<E, D>(p.kh + (keys + n) * D, p.rk[keys + n], dk, hh);
        if (mine) store_row<T, D>((T *)a.dk + tok * a.dks.token + head * a.dks.head, dk, hh);
    }
    if (GV && (WK == 1 || wave == 1)) {
        scale_up<DT>(dv, P == 2 ? 0.5f : 1.0f, ev);
        if (odd)
            add_odd<T, D>(dv, begin / 64 * 64, rows, lane, [&](int r) { return p.info[base + r].ed & 1; },
                          [&](int r) {
                              const int t = r / a.group;
                              return (const T *)a.dout + ((size_t)(pl.t0 + t) * a.Hq + head * a.group + r - t * a.group) * D;
                          },
                          [&](int r) { return r >= least; });
        if (mine) store_row<T, D>((T *)a.dv + tok * a.dvs.token + head * a.dvs.head, dv, hh);
    }
}

template <typename T, int D, int P, int WK>
__global__ __launch_bounds__(THREADS, WK > 1 || (sizeof(T) == 4 && D == 128) ? 1 : 2) void bwd_kernel(
    PackedArgs a, Planes<typename plane_of<T>::type> p)
{
    typedef typename plane_of<T>::type E;
    constexpr int N = Cut<E, D, WK>::TILE * Ops<E, D>::C;
    __shared__ u4 x0[N], x1[N], y0[N], y1[N];
    __shared__ f4 factors[THREADS / 64][32];
    __shared__ int wave_powers[THREADS / 64][64];
    f4 *const mine = factors[scalar(threadIdx.x / 64)];
    const int head = blockIdx.x % a.Hkv;
    const Place pl = scalar(p.places[blockIdx.x / a.Hkv]);
    if (pl.len == 0) return;
    if (pl.role == ROWS) {
        rows_block<T, D, P, WK>(a, p, head, pl, x0, x1, y0, y1, mine, wave_powers);
    } else if constexpr (WK == 1 && split_keys(D, sizeof(T) == 2)) {
        if (pl.role == DK) keys_block<T, D, P, DK, WK>(a, p, head, pl, x0, x1, y0, y1, mine, wave_powers);
        else keys_block<T, D, P, DV, WK>(a, p, head, pl, x0, x1, y0, y1, mine, wave_powers);
    } else {
        keys_block<T, D, P, KEYS, WK>(a, p, head, pl, x0, x1, y0, y1, mine, wave_powers);
    }
}

template <typename T, int D> static hipError_t launch_bwd(const PackedArgs &a, void *ws, hipStream_t st)
{
    typedef typename plane_of<T>::type E;
    const Planes<E> p = planes_at<E>(ws, a, D, 1);
    const long long blocks = (long long)p.n_places * a.Hkv;
    if (!grid_fits(blocks, THREADS)) return hipErrorInvalidConfiguration;
    const hipError_t e = prep<T, E>(a, p, D, 1, st);
    if (e != hipSuccess) return e;
    if constexpr (Cut<E, D, 4>::FITS) {
        if (p.cols == 32) {
            if (a.p == 2) bwd_kernel<T, D, 2, 4><<<(unsigned)blocks, THREADS, 0, st>>>(a, p);
            else bwd_kernel<T, D, 1, 4><<<(unsigned)blocks, THREADS, 0, st>>>(a, p);
            return hipGetLastError();
        }
    }
    if (a.p == 2) bwd_kernel<T, D, 2, 1><<<(unsigned)blocks, THREADS, 0, st>>>(a, p);
    else bwd_kernel<T, D, 1, 1><<<(unsigned)blocks, THREADS, 0, st>>>(a, p);
    return hipGetLastError();
}

template <typename T> static hipError_t launch_bwd_d(const PackedArgs &a, int D, void *ws, hipStream_t st)
{
    switch (D) {
    case 16: return launch_bwd<T, 16>(a, ws, st);
    case 32: return launch_bwd<T, 32>(a, ws, st);
    case 64: return launch_bwd<T, 64>(a, ws, st);
    default: return launch_bwd<T, 128>(a, ws, st);
    }
}

}  // namespace packed

hipError_t packed_bwd(const PackedArgs &a, int D, int is_bf16, void *ws, hipStream_t st)
{
    return is_bf16 ? packed::launch_bwd_d<bf16_t>(a, D, ws, st) : packed::launch_bwd_d<float>(a, D, ws, st);
}

}  // namespace fm
