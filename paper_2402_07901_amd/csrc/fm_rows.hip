// The rows around the attention: a projection's q, k, v rows (token after
// token, heads side by side) normed, rotated and laid out for the attention
// (forward, backward), or standardised as well and appended to a paged cache.
//
//     y = w x r, r = 1 / sqrt(mean x^2 + eps)      (w given)
//     z = R y                                      (fm_rows.h)
//     append: z^ = (z - mean z) / std z            (population, no epsilon)
// Backward: dy = R^T dz (dz summed over the heads that share the row),
//     dx = r (w dy - x r^2 mean(x w dy)),  dw = sum over rows of x r dy.
//
// Everything is in float32 registers between one read and one write, so HBM
// bounds it.  A lane holds 16 channels (two 16-byte loads in bf16); the
// D / 16 lanes of a row are neighbours and the rows of a wave are consecutive
// tokens of one head, so that the head-major side is one contiguous run per
// wave and the token-major side runs of D.  A lane keeps its token through a
// run of heads: cos and sin are read once for all of them.  bf16, norm and
// rotation: 4 x 8192 tokens, 16 heads of 64, forward 83 to 87 us (4.65 to 4.9 TB/s;
// cards differ), backward 110 to 116 us with the weights' gradients; 16384
// tokens of 32 and 8 heads of 128 appended in 82 to 89 us.  One token: 3.9 us, a launch.
#include <hip/hip_runtime.h>

#include "fm_internal.h"
#include "fm_rows.h"
#include "fm_serve.h"

namespace fm {
namespace {

using namespace rows;

constexpr int THREADS = 256;

// Which rows a workgroup takes of its tokens: heads [h0, h1) of q, k or v.
struct Run {
    int kind;   // 0 q, 1 k, 2 v
    int h0, h1;
};

// Heads are cut in runs of `per`: q's runs first, then k's, then v's.
__device__ __forceinline__ Run run_of(int y, int per, int Hq, int Hkv)
{
    const int nq = (Hq + per - 1) / per, nk = (Hkv + per - 1) / per;
    Run r;
    r.kind = y < nq ? 0 : y < nq + nk ? 1 : 2;
    r.h0 = per * (y - (r.kind == 0 ? 0 : r.kind == 1 ? nq : nq + nk));
    r.h1 = min(r.h0 + per, r.kind == 0 ? Hq : Hkv);
    return r;
}

long long runs(int per, int Hq, int Hkv)
{
    return (Hq + per - 1) / per + 2LL * ((Hkv + per - 1) / per);
}

// Heads per run: 8 share a lane's cos and sin; fewer where that leaves the
// GPU short of workgroups (4 per CU).
int heads_per_run(long long blocks, int Hq, int Hkv)
{
    int per = 8;
    while (per > 1 && blocks * runs(per, Hq, Hkv) < 1024) per /= 2;
    return per;
}

template <typename T, int D, bool APPEND>
__global__ __launch_bounds__(THREADS) void rows_kernel(RowsArgs a, int per)
{
    constexpr int L = D / 16, U = 4;
    const long long tokens = (long long)a.B * a.N;
    const long long lane = (long long)blockIdx.x * THREADS + threadIdx.x;
    const long long t = lane / L;
    const int c = (int)(lane % L);
    if (t >= tokens) return;   // whole rows: the row sums below stay among their own lanes
    const Run run = run_of(blockIdx.y, per, a.Hq, a.Hkv);
    const long long b = t / a.N, n = t - b * a.N;
    const int group = a.Hq / a.Hkv;

    const Strides st = run.kind == 0 ? a.qs : run.kind == 1 ? a.ks : a.vs;
    const T *src = (const T *)(run.kind == 0 ? a.q : run.kind == 1 ? a.k : a.v) + b * st.batch + n * st.token;
    T *dst = (T *)(run.kind == 0 ? a.oq : run.kind == 1 ? a.ok : a.ov);
    long long head, row;       // elements between heads, and where the token is in a head
    int copies = 1;
    if constexpr (!APPEND) {
        head = (long long)a.N * D;
        row = (b * a.Hq * (long long)a.N + n) * D;
        copies = run.kind == 0 ? 1 : group;
    } else if (run.kind == 0) {
        head = D;
        row = t * a.Hq * D;
    } else {
        const long long slot = a.slots[t];
        if (slot < 0 || slot >= (long long)a.pages << a.page_shift) return;
        head = a.cache.head;
        row = (slot >> a.page_shift) * a.cache.batch + (slot & ((1 << a.page_shift) - 1)) * a.cache.token;
    }

    const bool plain = run.kind == 2;
    Place at = {16 * c, 16 * c + 8, false};
    float cs[8], sn[8], w[16];
    const float *wp = run.kind == 0 ? a.rope.wq : a.rope.wk;
    if (!plain) {
        at = place_of(c, a.rope);
        if (at.turned) angles(a.rope, t, c, cs, sn);
        if (wp) {
            ld8(wp + at.a, w);
            ld8(wp + at.b, w + 8);
        }
    }
    for (int h = run.h0; h < run.h1; h += U) {
        float x[U][16];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (h + u < run.h1) {
                const T *p = src + (h + u) * st.head;
                ld8(p + at.a, x[u]);
                ld8(p + at.b, x[u] + 8);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (h + u >= run.h1) break;
            float *y = x[u];
            if (!plain) {
                if (wp) {
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) ss = fmaf(y[i], y[i], ss);
                    const float r = 1.0f / sqrtf(row_sum<L>(ss) * (1.0f / D) + a.rope.eps);
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] *= r * w[i];
                }
                if (at.turned) turn<false>(y, cs, sn, a.rope.interleaved);
                if constexpr (APPEND) {
                    float s = 0.f, v = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s += y[i];
                    const float mu = row_sum<L>(s) * (1.0f / D);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        y[i] -= mu;
                        v = fmaf(y[i], y[i], v);
                    }
                    const float r = 1.0f / sqrtf(row_sum<L>(v) * (1.0f / D));
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] *= r;
                }
            }
            T *o = dst + row + (long long)(h + u) * copies * head;
            for (int j = 0; j < copies; ++j, o += head) {
                st8(o + at.a, y);
                st8(o + at.b, y + 8);
            }
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void rope_bwd_kernel(RowsBwdArgs a, int per, float *partial)
{
    constexpr int L = D / 16;
    __shared__ float red[THREADS / 64][D];
    const long long tokens = (long long)a.B * a.N;
    const long long lane = (long long)blockIdx.x * THREADS + threadIdx.x;
    const int c = (int)(lane % L);
    const bool live = lane / L < tokens;
    const long long t = live ? lane / L : tokens - 1;
    const Run run = run_of(blockIdx.y, per, a.Hq, a.Hkv);
    const long long b = t / a.N, n = t - b * a.N;
    const int group = run.kind == 0 ? 1 : a.Hq / a.Hkv;

    const Strides st = run.kind == 0 ? a.dqs : run.kind == 1 ? a.dks : a.dvs;
    const Strides xs = run.kind == 0 ? a.qs : a.ks;
    const T *grad = (const T *)(run.kind == 0 ? a.gq : run.kind == 1 ? a.gk : a.gv);
    const T *xrow = (const T *)(run.kind == 0 ? a.q : a.k);
    T *dst = (T *)(run.kind == 0 ? a.dq : run.kind == 1 ? a.dk : a.dv) + b * st.batch + n * st.token;
    const float *wp = run.kind == 0 ? a.rope.wq : run.kind == 1 ? a.rope.wk : nullptr;

    const bool plain = run.kind == 2;
    Place at = {16 * c, 16 * c + 8, false};
    float cs[8], sn[8], w[16], dw[16];
    if (!plain) {
        at = place_of(c, a.rope);
        if (at.turned) angles(a.rope, t, c, cs, sn);
    }
    if (wp) {
        ld8(wp + at.a, w);
        ld8(wp + at.b, w + 8);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) dw[i] = 0.f;

    for (int h = run.h0; h < run.h1; ++h) {
        float d[16], x[16];
        const T *p = grad + ((b * a.Hq + (long long)h * group) * a.N + n) * D;
        ld8(p + at.a, d);
        ld8(p + at.b, d + 8);
        if (wp) {
            const T *xp = xrow + b * xs.batch + n * xs.token + h * xs.head;
            ld8(xp + at.a, x);
            ld8(xp + at.b, x + 8);
        }
        for (int j = 1; j < group; ++j) {
            float e[16];
            p += (long long)a.N * D;
            ld8(p + at.a, e);
            ld8(p + at.b, e + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] += e[i];
        }
        if (at.turned) turn<true>(d, cs, sn, a.rope.interleaved);
        if (wp) {
            float ss = 0.f, m = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
            const float r = 1.0f / sqrtf(row_sum<L>(ss) * (1.0f / D) + a.rope.eps);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] *= r;
                dw[i] = fmaf(d[i], x[i], dw[i]);
                d[i] *= w[i];
                m = fmaf(d[i], x[i], m);
            }
            m = row_sum<L>(m) * (1.0f / D);
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] = r * (d[i] - x[i] * m);
        }
        if (live) {
            T *o = dst + h * st.head;
            st8(o + at.a, d);
            st8(o + at.b, d + 8);
        }
    }
    if (!wp) return;
    // weight gradients: the rows of the wave (lanes with the same channels),
    // then the waves, in a fixed order; one partial row per workgroup
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float s = live ? dw[i] : 0.f;
        for (int o = L; o < 64; o *= 2) s += __shfl_xor(s, o);
        dw[i] = s;
    }
    const int wave = threadIdx.x / 64, l = threadIdx.x % 64;
    if (l < L) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            red[wave][at.a + i] = dw[i];
            red[wave][at.b + i] = dw[i + 8];
        }
    }
    __syncthreads();
    if (threadIdx.x < D) {
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < THREADS / 64; ++v) s += red[v][threadIdx.x];
        partial[((long long)blockIdx.y * gridDim.x + blockIdx.x) * D + threadIdx.x] = s;
    }
}

// dwq (block row 0) and dwk (1): sums of their partial rows, 16 channels of a
// workgroup, in double precision so that the order of a long sum does not show.
// Latency bounds it: a lane holds 4 channels, so that 256 rows stand side by
// side and 4 of a lane's are in flight, and only the waves' sums go through LDS
// (a lane with one channel and all of it through LDS: 2 to 3 us longer).
constexpr int SUM_THREADS = 1024;
__global__ __launch_bounds__(SUM_THREADS) void weight_sum_kernel(const float *partial, float *dwq, float *dwk,
                                                                 long long nq, long long nk, int D)
{
    constexpr int ROWS = SUM_THREADS / 4, U = 4;
    __shared__ double red[SUM_THREADS / 64][16];
    const bool keys = blockIdx.y;
    const long long rows = keys ? nk : nq;
    const float *p = partial + (keys ? nq * D : 0) + blockIdx.x * 16 + threadIdx.x % 4 * 4;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (long long r = threadIdx.x / 4; r < rows; r += ROWS * U) {
        float4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long ru = r + ROWS * u;
            x[u] = ru < rows ? *(const float4 *)(p + ru * D) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[0] += (double)x[u].x;
            s[1] += (double)x[u].y;
            s[2] += (double)x[u].z;
            s[3] += (double)x[u].w;
        }
    }
    for (int o = 4; o < 64; o *= 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] += __shfl_xor(s[i], o);
    }
    if (threadIdx.x % 64 < 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) red[threadIdx.x / 64][threadIdx.x % 4 * 4 + i] = s[i];
    }
    __syncthreads();
    if (threadIdx.x >= 16) return;
    double sum = 0.0;
#pragma unroll
    for (int v = 0; v < SUM_THREADS / 64; ++v) sum += red[v][threadIdx.x];
    (keys ? dwk : dwq)[blockIdx.x * 16 + threadIdx.x] = (float)sum;
}

long long token_blocks(long long tokens, int D) { return (tokens * (D / 16) + THREADS - 1) / THREADS; }

bool rows_fit(long long blocks, long long y)
{
    return grid_fits(blocks, THREADS) && y <= 65535;
}

template <bool APPEND> hipError_t rows_launch(const RowsArgs &a, int D, int is_bf16, hipStream_t st)
{
    const long long blocks = token_blocks((long long)a.B * a.N, D);
    const int per = heads_per_run(blocks, a.Hq, a.Hkv);
    const long long y = runs(per, a.Hq, a.Hkv);
    if (!rows_fit(blocks, y)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks, (unsigned)y);
#define FM_ROWS(DD)                                                                               \
    case DD:                                                                                      \
        if (is_bf16) rows_kernel<bf16_t, DD, APPEND><<<grid, THREADS, 0, st>>>(a, per);           \
        else rows_kernel<float, DD, APPEND><<<grid, THREADS, 0, st>>>(a, per);                    \
        break
    switch (D) {
        FM_ROWS(16);
        FM_ROWS(32);
        FM_ROWS(64);
        FM_ROWS(128);
    }
#undef FM_ROWS
    return hipGetLastError();
}

}  // namespace

hipError_t rope_fwd(const RowsArgs &a, int D, int is_bf16, hipStream_t st)
{
    return rows_launch<false>(a, D, is_bf16, st);
}

hipError_t cache_append(const RowsArgs &a, int D, int is_bf16, hipStream_t st)
{
    return rows_launch<true>(a, D, is_bf16, st);
}

size_t rope_bwd_workspace(long long tokens, int Hq, int Hkv, int D, int norm)
{
    if (!norm) return 0;
    const long long blocks = token_blocks(tokens, D);
    const int per = heads_per_run(blocks, Hq, Hkv);
    return (size_t)(blocks * runs(per, Hq, Hkv)) * D * sizeof(float);
}

hipError_t rope_bwd(const RowsBwdArgs &a, int D, int is_bf16, void *ws, hipStream_t st)
{
    const long long blocks = token_blocks((long long)a.B * a.N, D);
    const int per = heads_per_run(blocks, a.Hq, a.Hkv);
    const long long y = runs(per, a.Hq, a.Hkv);
    if (!rows_fit(blocks, y)) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks, (unsigned)y);
    float *partial = (float *)ws;
#define FM_ROWS(DD)                                                                               \
    case DD:                                                                                      \
        if (is_bf16) rope_bwd_kernel<bf16_t, DD><<<grid, THREADS, 0, st>>>(a, per, partial);      \
        else rope_bwd_kernel<float, DD><<<grid, THREADS, 0, st>>>(a, per, partial);               \
        break
    switch (D) {
        FM_ROWS(16);
        FM_ROWS(32);
        FM_ROWS(64);
        FM_ROWS(128);
    }
#undef FM_ROWS
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.rope.wq) return e;
    const long long nq = blocks * ((a.Hq + per - 1) / per), nk = blocks * ((a.Hkv + per - 1) / per);
    weight_sum_kernel<<<dim3(D / 16, 2), SUM_THREADS, 0, st>>>(partial, a.dwq, a.dwk, nq, nk, D);
    return hipGetLastError();
}

}  // namespace fm
