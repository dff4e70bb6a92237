// C ABI of the row kernels and the paged attention: host-side validation,
// workspace sizing and launch.  Every check runs before anything is enqueued.
#include <limits.h>
#include <stdint.h>
#include <string.h>

#include "../../include/fastmax.h"
#include "fm_internal.h"
#include "fm_serve.h"

namespace fm {
int code_of(hipError_t e);
}

namespace {

constexpr int NO_WINDOW = 1 << 30;   // wider than any sequence
constexpr int CODES = 2;             // 8-bit rows, beside the fastmax_dtype_t

bool supported_d(int D) { return D == 16 || D == 32 || D == 64 || D == 128; }
bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

int dt_bits(const fastmax_dtype_t *dt)   // any int may come from a C caller
{
    int v;
    memcpy(&v, dt, sizeof v);
    return v;
}

// tokens: B * N or T
int check_sizes(long long tokens, int Hq, int Hkv, int D, int dt)
{
    if (tokens < 1 || tokens > (1LL << 40) || Hq < 1 || Hkv < 1 || Hq > (1 << 16) || Hq % Hkv) return FASTMAX_EINVAL;
    if (dt != FASTMAX_F32 && dt != FASTMAX_BF16) return FASTMAX_EINVAL;
    if (!supported_d(D)) return FASTMAX_EUNSUPPORTED;
    if ((unsigned __int128)tokens * Hq * D >= ((unsigned __int128)1 << 62)) return FASTMAX_EINVAL;
    return FASTMAX_OK;
}

int check_rope(const fastmax_rope_t *r, int D, fm::Rope *out)
{
    if (!r) return FASTMAX_ENULL;
    if (r->rot < 0 || r->rot > D || r->rot % 16) return FASTMAX_EINVAL;
    if (r->interleaved != 0 && r->interleaved != 1) return FASTMAX_EINVAL;
    if (!(r->eps >= 0.0f) || r->eps > 1e30f) return FASTMAX_EINVAL;
    if (!r->wq != !r->wk) return FASTMAX_ENULL;
    if (!aligned(r->wq, 16) || !aligned(r->wk, 16)) return FASTMAX_EALIGN;
    out->half = r->rot / 2;
    out->axes = 1;
    out->end[0] = out->end[1] = out->end[2] = INT_MAX;
    if (r->rot) {
        if (r->axes < 1 || r->axes > 4 || r->table_rows < 1) return FASTMAX_EINVAL;
        if (r->axes > 1) {
            int sum = 0;
            for (int i = 0; i < r->axes; ++i) {
                if (r->sections[i] < 0 || r->sections[i] > out->half) return FASTMAX_EINVAL;
                sum += r->sections[i];
                if (i < r->axes - 1) out->end[i] = sum;
            }
            if (sum != out->half) return FASTMAX_EINVAL;
            out->axes = r->axes;
        }
        if (!r->cos || !r->sin || !r->pos) return FASTMAX_ENULL;
        if (!aligned(r->cos, 16) || !aligned(r->sin, 16) || !aligned(r->pos, 4)) return FASTMAX_EALIGN;
    }
    out->cos = r->cos;
    out->sin = r->sin;
    out->pos = r->pos;
    out->table_rows = r->table_rows;
    out->interleaved = r->interleaved;
    out->wq = r->wq;
    out->wk = r->wk;
    out->eps = r->eps;
    return FASTMAX_OK;
}

// Strides of token rows [B, N, H, D]: contiguous when none are given; rows
// stay 16-byte aligned; `rows_apart`: no two rows may share memory (outputs).
int check_strides(const fastmax_strides_t *s, int B, int N, int H, int D, int dt, bool rows_apart, fm::Strides *out)
{
    if (!s) {
        *out = {(long long)N * H * D, (long long)H * D, D};
        return FASTMAX_OK;
    }
    const long long st[3] = {B > 1 ? s->batch : 0, N > 1 ? s->token : 0, H > 1 ? s->head : 0};
    const int n[3] = {B, N, H};
    for (int i = 0; i < 3; ++i) {
        if (st[i] < 0 || st[i] > (1LL << 46)) return FASTMAX_EINVAL;
        if (rows_apart && n[i] > 1 && st[i] < D) return FASTMAX_EINVAL;
        if (st[i] % (dt == CODES ? 16 : dt == FASTMAX_BF16 ? 8 : 4)) return FASTMAX_EALIGN;
    }
    *out = {st[0], st[1], st[2]};
    return FASTMAX_OK;
}

int check_cache(const fastmax_strides_t *s, int Hkv, int D, int pages, int page_size, int dt, bool rows_apart,
                fm::Strides *out, int *shift)
{
    if (pages < 1 || page_size < 16 || page_size > 1024 || (page_size & (page_size - 1))) return FASTMAX_EINVAL;
    *shift = __builtin_ctz((unsigned)page_size);
    if (!s) {
        *out = {(long long)Hkv * page_size * D, D, (long long)page_size * D};
        return FASTMAX_OK;
    }
    if (s->token > (1 << 26)) return FASTMAX_EINVAL;   // a tile's places are 32-bit offsets
    return check_strides(s, pages, page_size, Hkv, D, dt, rows_apart, out);
}

int check_ptrs(const void *const *p, int n)
{
    for (int i = 0; i < n; ++i)
        if (!p[i]) return FASTMAX_ENULL;
    for (int i = 0; i < n; ++i)
        if (!aligned(p[i], 16)) return FASTMAX_EALIGN;
    return FASTMAX_OK;
}

const fastmax_strides_t *nth(const fastmax_strides_t *s, int i) { return s ? s + i : nullptr; }

// The three token-row tensors of a call.
int check_rows(const fastmax_strides_t *s, int n, int B, int N, int Hq, int Hkv, int D, int dt, bool rows_apart,
               fm::Strides *q, fm::Strides *k, fm::Strides *v)
{
    fm::Strides *out[3] = {q, k, v};
    for (int i = 0; i < n; ++i) {
        const int rc = check_strides(nth(s, i), B, N, i ? Hkv : Hq, D, dt, rows_apart, out[i]);
        if (rc != FASTMAX_OK) return rc;
    }
    return FASTMAX_OK;
}

// Sizes of a paged call that the workspace depends on.
int check_paged(int S, int T, int Hq, int Hkv, int D, int max_q, int max_len, int window, int sinks, int dt)
{
    const int rc = check_sizes(T, Hq, Hkv, D, dt);
    if (rc != FASTMAX_OK) return rc;
    if (S < 1 || S > 65535 || max_q < 1 || max_q > T || max_len < 1 || max_len > (1 << 30)) return FASTMAX_EINVAL;
    if (window < 0 || sinks < 0 || (long long)T * Hq > INT_MAX / 2) return FASTMAX_EINVAL;
    return FASTMAX_OK;
}

// The append's arguments; cache_dt: what the cache holds.
int check_append(fm::RowsArgs *a, const void *q, const void *k, const void *v, const fastmax_strides_t *strides,
                 void *q_out, void *k_cache, void *v_cache, const fastmax_strides_t *cache, const int64_t *slots,
                 int T, int Hq, int Hkv, int D, int pages, int page_size, const fastmax_rope_t *rope, int dt,
                 int cache_dt, hipStream_t stream)
{
    int rc = check_sizes(T, Hq, Hkv, D, dt);
    if (rc != FASTMAX_OK) return rc;
    if ((rc = check_rope(rope, D, &a->rope)) != FASTMAX_OK) return rc;
    if ((rc = check_rows(strides, 3, 1, T, Hq, Hkv, D, dt, false, &a->qs, &a->ks, &a->vs)) != FASTMAX_OK) return rc;
    if ((rc = check_cache(cache, Hkv, D, pages, page_size, cache_dt, true, &a->cache, &a->page_shift)) != FASTMAX_OK)
        return rc;
    const void *ptrs[] = {q, k, v, q_out, k_cache, v_cache};
    if ((rc = check_ptrs(ptrs, 6)) != FASTMAX_OK) return rc;
    if (!slots) return FASTMAX_ENULL;
    if (!aligned(slots, 8)) return FASTMAX_EALIGN;
    if ((rc = fm::check_stream(stream)) != FASTMAX_OK) return rc;
    a->q = q, a->k = k, a->v = v, a->oq = q_out, a->ok = k_cache, a->ov = v_cache;
    a->B = 1, a->N = T, a->Hq = Hq, a->Hkv = Hkv;
    a->slots = slots, a->pages = pages;
    return FASTMAX_OK;
}

// The plan of a paged call whose sizes are checked.
fm::PagedPlan plan_of(bool q8, int S, int Hq, int Hkv, int D, int max_q, int max_len, int window, int sinks, int dt)
{
    const int wide = window && window < NO_WINDOW ? window : NO_WINDOW;
    const int bf16 = dt == FASTMAX_BF16;
    if (q8) return fm::paged_q8_plan(S, Hq, Hkv, D, max_q, max_len, wide, sinks);
    return fm::paged_plan(S, Hq, Hkv, D, bf16, max_q, max_len, wide, sinks, !bf16 && D == 128 ? 32 : 64);
}

// The paged attention's arguments; cache_dt: what the cache holds.
int check_paged_call(fm::PagedArgs *a, fm::PagedPlan *plan, const void *q, const fastmax_strides_t *q_strides,
                     const void *k_cache, const void *v_cache, const fastmax_strides_t *cache, const int32_t *table,
                     const int32_t *lens, const int32_t *q_start, void *out, int S, int T, int Hq, int Hkv, int D,
                     int pages, int page_size, int table_cols, int max_q, int max_len, int p, float qk_scale,
                     int window, int sinks, int dt, int cache_dt, void *workspace, size_t workspace_bytes,
                     hipStream_t stream)
{
    int rc = check_paged(S, T, Hq, Hkv, D, max_q, max_len, window, sinks, dt);
    if (rc != FASTMAX_OK) return rc;
    if (p != 1 && p != 2) return FASTMAX_EINVAL;
    if (!(qk_scale > 0.0f && qk_scale <= 1.0f)) return FASTMAX_EINVAL;
    if (!q_start && (T != S || max_q != 1)) return FASTMAX_EINVAL;
    if ((rc = check_cache(cache, Hkv, D, pages, page_size, cache_dt, false, &a->cache, &a->page_shift)) != FASTMAX_OK)
        return rc;
    if (table_cols < 1 || (long long)table_cols * page_size > (1 << 30)) return FASTMAX_EINVAL;
    fm::Strides qs;
    if ((rc = check_strides(q_strides, 1, T, Hq, D, dt, false, &qs)) != FASTMAX_OK) return rc;
    const void *ptrs[] = {q, k_cache, v_cache, out};
    if ((rc = check_ptrs(ptrs, 4)) != FASTMAX_OK) return rc;
    if (!table || !lens) return FASTMAX_ENULL;
    if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(q_start, 4)) return FASTMAX_EALIGN;
    *plan = plan_of(cache_dt == CODES, S, Hq, Hkv, D, max_q, max_len, window, sinks, dt);
    const size_t need = fm::paged_workspace(*plan, T, Hq, D);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FASTMAX_EWORKSPACE;
    if (workspace && !aligned(workspace, 16)) return FASTMAX_EALIGN;
    if ((rc = fm::check_stream(stream)) != FASTMAX_OK) return rc;
    a->q = q, a->k = k_cache, a->v = v_cache, a->out = out;
    a->q_token = qs.token, a->q_head = qs.head;
    a->table = table, a->lens = lens, a->q_start = q_start;
    a->S = S, a->T = T, a->Hq = Hq, a->Hkv = Hkv, a->group = Hq / Hkv;
    a->pages = pages, a->table_cols = table_cols;
    a->window = window && window < NO_WINDOW ? window : NO_WINDOW, a->sinks = sinks;
    a->c1 = qk_scale, a->c2 = p == 2 ? 0.5f * qk_scale * qk_scale : 0.0f;
    return FASTMAX_OK;
}

size_t paged_bytes(bool q8, int S, int T, int Hq, int Hkv, int D, int max_q, int max_len, int window, int sinks, int dt)
{
    if (check_paged(S, T, Hq, Hkv, D, max_q, max_len, window, sinks, dt) != FASTMAX_OK) return 0;
    return fm::paged_workspace(plan_of(q8, S, Hq, Hkv, D, max_q, max_len, window, sinks, dt), T, Hq, D);
}

// Sequences and rows of a packed call (a row's number is an int, with room for a
// workgroup's beyond the last).
bool packed_fits(int S, int T, int Hq) { return S >= 1 && S <= (1 << 20) && (long long)T * Hq <= 1 << 30; }

// The packed attention's arguments (backward: with dout, dq, dk, dv).
int check_packed(fm::PackedArgs *a, const void *q, const void *k, const void *v, const fastmax_strides_t *strides,
                 const int32_t *starts, const void *out, const float *g, int S, int T, int Hq, int Hkv, int D, int p,
                 int causal, float qk_scale, int dt)
{
    int rc = check_sizes(T, Hq, Hkv, D, dt);
    if (rc != FASTMAX_OK) return rc;
    if (!packed_fits(S, T, Hq)) return FASTMAX_EINVAL;
    if ((p != 1 && p != 2) || (causal != 0 && causal != 1)) return FASTMAX_EINVAL;
    if (!(qk_scale > 0.0f && qk_scale <= 1.0f)) return FASTMAX_EINVAL;
    if ((rc = check_rows(strides, 3, 1, T, Hq, Hkv, D, dt, false, &a->qs, &a->ks, &a->vs)) != FASTMAX_OK) return rc;
    const void *ptrs[] = {q, k, v, out};
    if ((rc = check_ptrs(ptrs, 4)) != FASTMAX_OK) return rc;
    if (!starts) return FASTMAX_ENULL;
    if (!aligned(starts, 4) || !aligned(g, 16)) return FASTMAX_EALIGN;
    a->q = q, a->k = k, a->v = v, a->starts = starts, a->out = (void *)out, a->g = (float *)g;
    a->S = S, a->T = T, a->Hq = Hq, a->Hkv = Hkv, a->group = Hq / Hkv, a->p = p, a->causal = causal;
    a->tau = qk_scale;
    return FASTMAX_OK;
}

int check_workspace(const void *workspace, size_t bytes, size_t need)
{
    if (need > 0 && (!workspace || bytes < need)) return FASTMAX_EWORKSPACE;
    return aligned(workspace, 16) ? FASTMAX_OK : FASTMAX_EALIGN;
}

}  // namespace

extern "C" {

int fastmax_rope_fwd(const void *q, const void *k, const void *v, const fastmax_strides_t *strides, void *oq,
                     void *ok, void *ov, int B, int N, int Hq, int Hkv, int D, const fastmax_rope_t *rope,
                     fastmax_dtype_t dt_arg, hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg);
    if (B < 1 || N < 1) return FASTMAX_EINVAL;
    int rc = check_sizes((long long)B * N, Hq, Hkv, D, dt);
    if (rc != FASTMAX_OK) return rc;
    fm::RowsArgs a = {};
    if ((rc = check_rope(rope, D, &a.rope)) != FASTMAX_OK) return rc;
    if ((rc = check_rows(strides, 3, B, N, Hq, Hkv, D, dt, false, &a.qs, &a.ks, &a.vs)) != FASTMAX_OK) return rc;
    const void *ptrs[] = {q, k, v, oq, ok, ov};
    if ((rc = check_ptrs(ptrs, 6)) != FASTMAX_OK) return rc;
    if ((rc = fm::check_stream(stream)) != FASTMAX_OK) return rc;
    a.q = q, a.k = k, a.v = v, a.oq = oq, a.ok = ok, a.ov = ov;
    a.B = B, a.N = N, a.Hq = Hq, a.Hkv = Hkv;
    return fm::code_of(fm::rope_fwd(a, D, dt == FASTMAX_BF16, stream));
}

size_t fastmax_rope_workspace_bytes(int B, int N, int Hq, int Hkv, int D, int norm)
{
    if (B < 1 || N < 1 || check_sizes((long long)B * N, Hq, Hkv, D, FASTMAX_F32) != FASTMAX_OK) return 0;
    return fm::rope_bwd_workspace((long long)B * N, Hq, Hkv, D, norm);
}

int fastmax_rope_bwd(const void *q, const void *k, const fastmax_strides_t *strides, const void *gq,
                     const void *gk, const void *gv, void *dq, void *dk, void *dv,
                     const fastmax_strides_t *dstrides, float *dwq, float *dwk, int B, int N, int Hq, int Hkv,
                     int D, const fastmax_rope_t *rope, fastmax_dtype_t dt_arg, void *workspace,
                     size_t workspace_bytes, hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg);
    if (B < 1 || N < 1) return FASTMAX_EINVAL;
    int rc = check_sizes((long long)B * N, Hq, Hkv, D, dt);
    if (rc != FASTMAX_OK) return rc;
    fm::RowsBwdArgs a = {};
    if ((rc = check_rope(rope, D, &a.rope)) != FASTMAX_OK) return rc;
    fm::Strides none;
    if ((rc = check_rows(strides, 2, B, N, Hq, Hkv, D, dt, false, &a.qs, &a.ks, &none)) != FASTMAX_OK) return rc;
    if ((rc = check_rows(dstrides, 3, B, N, Hq, Hkv, D, dt, true, &a.dqs, &a.dks, &a.dvs)) != FASTMAX_OK) return rc;
    const bool norm = rope->wq != nullptr;
    const void *ptrs[] = {gq, gk, gv, dq, dk, dv, q, k, dwq, dwk};
    if ((rc = check_ptrs(ptrs, norm ? 10 : 6)) != FASTMAX_OK) return rc;
    const size_t need = fm::rope_bwd_workspace((long long)B * N, Hq, Hkv, D, norm);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FASTMAX_EWORKSPACE;
    if (workspace && !aligned(workspace, 16)) return FASTMAX_EALIGN;
    if ((rc = fm::check_stream(stream)) != FASTMAX_OK) return rc;
    a.q = q, a.k = k, a.gq = gq, a.gk = gk, a.gv = gv, a.dq = dq, a.dk = dk, a.dv = dv, a.dwq = dwq, a.dwk = dwk;
    a.B = B, a.N = N, a.Hq = Hq, a.Hkv = Hkv;
    return fm::code_of(fm::rope_bwd(a, D, dt == FASTMAX_BF16, workspace, stream));
}

int fastmax_cache_append(const void *q, const void *k, const void *v, const fastmax_strides_t *strides,
                         void *q_out, void *k_cache, void *v_cache, const fastmax_strides_t *cache,
                         const int64_t *slots, int T, int Hq, int Hkv, int D, int pages, int page_size,
                         const fastmax_rope_t *rope, fastmax_dtype_t dt_arg, hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg);
    fm::RowsArgs a = {};
    const int rc = check_append(&a, q, k, v, strides, q_out, k_cache, v_cache, cache, slots, T, Hq, Hkv, D, pages,
                                page_size, rope, dt, dt, stream);
    return rc != FASTMAX_OK ? rc : fm::code_of(fm::cache_append(a, D, dt == FASTMAX_BF16, stream));
}

int fastmax_cache_append_q8(const void *q, const void *k, const void *v, const fastmax_strides_t *strides,
                            void *q_out, int8_t *k_cache, int8_t *v_cache, float *k_scale, float *v_scale,
                            const fastmax_strides_t *cache, const int64_t *slots, int T, int Hq, int Hkv, int D,
                            int pages, int page_size, const fastmax_rope_t *rope, fastmax_dtype_t dt_arg,
                            hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg);
    const void *scales[] = {k_scale, v_scale};
    fm::RowsArgs a = {};
    int rc = check_append(&a, q, k, v, strides, q_out, k_cache, v_cache, cache, slots, T, Hq, Hkv, D, pages,
                          page_size, rope, dt, CODES, stream);
    if (rc == FASTMAX_OK) rc = check_ptrs(scales, 2);
    if (rc != FASTMAX_OK) return rc;
    a.k_scale = k_scale, a.v_scale = v_scale;
    return fm::code_of(fm::cache_append_q8(a, D, dt == FASTMAX_BF16, stream));
}

int fastmax_cache_read_q8(const int8_t *k_cache, const int8_t *v_cache, const float *k_scale, const float *v_scale,
                          const fastmax_strides_t *cache, const int64_t *slots, void *k, void *v, int T, int Hkv,
                          int D, int pages, int page_size, fastmax_dtype_t dt_arg, hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg);
    int rc = check_sizes(T, Hkv, Hkv, D, dt);
    if (rc != FASTMAX_OK) return rc;
    fm::ReadArgs a = {};
    if ((rc = check_cache(cache, Hkv, D, pages, page_size, CODES, false, &a.cache, &a.page_shift)) != FASTMAX_OK)
        return rc;
    const void *ptrs[] = {k_cache, v_cache, k_scale, v_scale, k, v};
    if ((rc = check_ptrs(ptrs, 6)) != FASTMAX_OK) return rc;
    if (!slots) return FASTMAX_ENULL;
    if (!aligned(slots, 8)) return FASTMAX_EALIGN;
    if ((rc = fm::check_stream(stream)) != FASTMAX_OK) return rc;
    a.k = k_cache, a.v = v_cache, a.k_scale = k_scale, a.v_scale = v_scale;
    a.slots = slots, a.ok = k, a.ov = v;
    a.T = T, a.Hkv = Hkv, a.pages = pages;
    return fm::code_of(fm::cache_read_q8(a, D, dt == FASTMAX_BF16, stream));
}

size_t fastmax_paged_workspace_bytes(int S, int T, int Hq, int Hkv, int D, int max_q, int max_len, int window,
                                     int sinks, fastmax_dtype_t dt_arg)
{
    return paged_bytes(false, S, T, Hq, Hkv, D, max_q, max_len, window, sinks, dt_bits(&dt_arg));
}

size_t fastmax_paged_q8_workspace_bytes(int S, int T, int Hq, int Hkv, int D, int max_q, int max_len, int window,
                                        int sinks, fastmax_dtype_t dt_arg)
{
    return paged_bytes(true, S, T, Hq, Hkv, D, max_q, max_len, window, sinks, dt_bits(&dt_arg));
}

int fastmax_paged_fwd(const void *q, const fastmax_strides_t *q_strides, const void *k_cache, const void *v_cache,
                      const fastmax_strides_t *cache, const int32_t *table, const int32_t *lens,
                      const int32_t *q_start, void *out, int S, int T, int Hq, int Hkv, int D, int pages,
                      int page_size, int table_cols, int max_q, int max_len, int p, float qk_scale, int window,
                      int sinks, fastmax_dtype_t dt_arg, void *workspace, size_t workspace_bytes,
                      hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg);
    fm::PagedArgs a = {};
    fm::PagedPlan plan;
    const int rc = check_paged_call(&a, &plan, q, q_strides, k_cache, v_cache, cache, table, lens, q_start, out, S, T,
                                    Hq, Hkv, D, pages, page_size, table_cols, max_q, max_len, p, qk_scale, window,
                                    sinks, dt, dt, workspace, workspace_bytes, stream);
    return rc != FASTMAX_OK ? rc : fm::code_of(fm::paged_fwd(a, plan, D, dt == FASTMAX_BF16, workspace, stream));
}

int fastmax_paged_fwd_q8(const void *q, const fastmax_strides_t *q_strides, const int8_t *k_cache,
                         const int8_t *v_cache, const float *k_scale, const float *v_scale,
                         const fastmax_strides_t *cache, const int32_t *table, const int32_t *lens,
                         const int32_t *q_start, void *out, int S, int T, int Hq, int Hkv, int D, int pages,
                         int page_size, int table_cols, int max_q, int max_len, int p, float qk_scale, int window,
                         int sinks, fastmax_dtype_t dt_arg, void *workspace, size_t workspace_bytes,
                         hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg);
    const void *scales[] = {k_scale, v_scale};
    fm::PagedArgs a = {};
    fm::PagedPlan plan;
    int rc = check_paged_call(&a, &plan, q, q_strides, k_cache, v_cache, cache, table, lens, q_start, out, S, T, Hq,
                              Hkv, D, pages, page_size, table_cols, max_q, max_len, p, qk_scale, window, sinks, dt,
                              CODES, workspace, workspace_bytes, stream);
    if (rc == FASTMAX_OK) rc = check_ptrs(scales, 2);
    if (rc != FASTMAX_OK) return rc;
    a.k_scale = k_scale, a.v_scale = v_scale;
    return fm::code_of(fm::paged_q8_fwd(a, plan, D, dt == FASTMAX_BF16, workspace, stream));
}

size_t fastmax_packed_workspace_bytes(int S, int T, int Hq, int Hkv, int D, fastmax_dtype_t dt_arg, int backward)
{
    const int dt = dt_bits(&dt_arg);
    if (check_sizes(T, Hq, Hkv, D, dt) != FASTMAX_OK || !packed_fits(S, T, Hq)) return 0;
    return fm::packed_workspace(S, T, Hq, Hkv, D, dt == FASTMAX_BF16, backward);
}

int fastmax_packed_fwd(const void *q, const void *k, const void *v, const fastmax_strides_t *strides,
                       const int32_t *starts, void *out, float *g, int S, int T, int Hq, int Hkv, int D, int p,
                       int causal, float qk_scale, fastmax_dtype_t dt_arg, void *workspace, size_t workspace_bytes,
                       hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg), bf16 = dt == FASTMAX_BF16;
    fm::PackedArgs a = {};
    int rc = check_packed(&a, q, k, v, strides, starts, out, g, S, T, Hq, Hkv, D, p, causal, qk_scale, dt);
    if (rc != FASTMAX_OK) return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, fm::packed_workspace(S, T, Hq, Hkv, D, bf16, 0))) != FASTMAX_OK)
        return rc;
    if ((rc = fm::check_stream(stream)) != FASTMAX_OK) return rc;
    return fm::code_of(fm::packed_fwd(a, D, bf16, workspace, stream));
}

int fastmax_packed_bwd(const void *q, const void *k, const void *v, const fastmax_strides_t *strides,
                       const int32_t *starts, const void *out, const void *dout, const float *g, void *dq, void *dk,
                       void *dv, const fastmax_strides_t *dstrides, int S, int T, int Hq, int Hkv, int D, int p,
                       int causal, float qk_scale, fastmax_dtype_t dt_arg, void *workspace, size_t workspace_bytes,
                       hipStream_t stream)
{
    const int dt = dt_bits(&dt_arg), bf16 = dt == FASTMAX_BF16;
    fm::PackedArgs a = {};
    int rc = check_packed(&a, q, k, v, strides, starts, out, g, S, T, Hq, Hkv, D, p, causal, qk_scale, dt);
    if (rc != FASTMAX_OK) return rc;
    if ((rc = check_rows(dstrides, 3, 1, T, Hq, Hkv, D, dt, true, &a.dqs, &a.dks, &a.dvs)) != FASTMAX_OK) return rc;
    const void *ptrs[] = {g, dout, dq, dk, dv};
    if ((rc = check_ptrs(ptrs, 5)) != FASTMAX_OK) return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, fm::packed_workspace(S, T, Hq, Hkv, D, bf16, 1))) != FASTMAX_OK)
        return rc;
    if ((rc = fm::check_stream(stream)) != FASTMAX_OK) return rc;
    a.dout = dout, a.dq = dq, a.dk = dk, a.dv = dv;
    return fm::code_of(fm::packed_bwd(a, D, bf16, workspace, stream));
}

}  // extern "C"
