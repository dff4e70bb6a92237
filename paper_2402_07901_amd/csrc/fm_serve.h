// Internal launch interface of the row kernels (fm_rows.hip) and the paged
// attention (fm_paged.hip); argument checks are api_serve.cpp's.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace fm {

// Rotation and norm of query and key rows (fastmax_rope_t, checked).
struct Rope {
    const float *cos, *sin;   // [table_rows, half]
    const int32_t *pos;       // [tokens, axes]
    int table_rows, half, axes, interleaved;
    int end[3];               // axis a's pairs end before end[a]; the last axis takes the rest
    const float *wq, *wk;     // norm weights [D], both or neither
    float eps;
};

// Strides in elements; D contiguous.
struct Strides {
    long long batch, token, head;
};

struct RowsArgs {
    const void *q, *k, *v;         // token rows
    Strides qs, ks, vs;
    void *oq, *ok, *ov;            // [B, Hq, N, D]; append: q^ [T, Hq, D] and the caches
    int B, N, Hq, Hkv;
    Rope rope;
    // append
    Strides cache;                 // batch: page, token: slot in the page, head
    const int64_t *slots;
    int pages, page_shift;
};
hipError_t rope_fwd(const RowsArgs &a, int D, int is_bf16, hipStream_t st);
hipError_t cache_append(const RowsArgs &a, int D, int is_bf16, hipStream_t st);

struct RowsBwdArgs {
    const void *q, *k;             // the forward's rows (norm only)
    Strides qs, ks;
    const void *gq, *gk, *gv;      // upstream gradients [B, Hq, N, D]
    void *dq, *dk, *dv;            // token rows
    Strides dqs, dks, dvs;
    float *dwq, *dwk;              // [D] (norm only)
    int B, N, Hq, Hkv;
    Rope rope;
};
size_t rope_bwd_workspace(long long tokens, int Hq, int Hkv, int D, int norm);
hipError_t rope_bwd(const RowsBwdArgs &a, int D, int is_bf16, void *ws, hipStream_t st);

struct PagedArgs {
    const void *q, *k, *v;
    void *out;                     // [T, Hq, D]
    long long q_token, q_head;     // strides of q
    Strides cache;                 // batch: page, token: slot in the page, head
    const int32_t *table, *lens, *q_start;
    int S, T, Hq, Hkv, group, pages, table_cols, page_shift;
    int window, sinks;             // window 2^30: none
    float c1, c2;                  // weight 1 + s (c1 + c2 s) of the raw product s; c2 is 0 for first order
};
// How a call is cut: rows of a (sequence, key head) in tiles, keys in splits.
struct PagedPlan {
    bool chunk_kernel;             // fm_paged_chunk.hip, else fm_paged.hip
    int rows;                      // rows of a row tile
    int waves;                     // of a workgroup (fm_paged.hip)
    int tiles;                     // row tiles in the grid
    int chunk;                     // key tiles of 16 per split
    int splits;
};
PagedPlan paged_plan(int S, int Hq, int Hkv, int D, int is_bf16, int max_q, int max_len, int window,
                     int sinks);
size_t paged_workspace(const PagedPlan &plan, int T, int Hq, int D);
hipError_t paged_fwd(const PagedArgs &a, const PagedPlan &plan, int D, int is_bf16, void *ws,
                     hipStream_t st);
constexpr int CHUNK_ROWS = 128;    // rows of a workgroup of the chunk kernel
hipError_t paged_chunk(const PagedArgs &a, const PagedPlan &plan, int D, int is_bf16, float *part,
                       hipStream_t st);

}  // namespace fm
