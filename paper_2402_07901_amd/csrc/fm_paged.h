// What the paged attention kernels share: which keys a row of queries sees, in
// tiles of 16, and where a sequence's rows are.
//
// Every key that is loaded is one that some row of the tile sees: lanes whose
// key is past the end, or in the gap behind the window, read such a key
// instead and get weight 0, so what lies in unused or evicted slots never
// enters a product.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fm_serve.h"

namespace fm {
namespace paged {

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

// Whether a query at position pos sees a key of a page that is not there, among
// the key tiles [begin, end): asked only once such a page was met.
__device__ __forceinline__ bool sees_bad_page(const PagedArgs &a, const int32_t *table, const Span &sp, int begin,
                                              int end, int pos)
{
    bool bad = false;
#pragma unroll 1
    for (int i = begin; i < end; ++i) {
        const int n0 = sp.tile(i) * KT;
        if ((unsigned)table[n0 >> a.page_shift] < (unsigned)a.pages) continue;
        bad |= n0 <= pos && (min(n0 + KT - 1, pos) > pos - a.window || n0 < a.sinks);
    }
    return bad;
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

// A value that is the same in every lane, in a scalar register (divisions
// leave it in a vector register, and all that follows with it).
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Span scalar(Span s)
{
    return Span{scalar(s.end), scalar(s.low_key), scalar(s.sinks), scalar(s.sink_tiles), scalar(s.low), scalar(s.tiles)};
}

}  // namespace paged
}  // namespace fm
