// Internal interface of the paged bf16 KV cache and of the norm and rotation of
// queries and keys: the host checks (kvp_host.cpp) and the kernels
// (qk_rotate.hip, kvp_attend.hip).  Not part of the public ABI.
#pragma once

#include "internal.h"

namespace cap {

// A grid of n workgroups of 256 (a launch counts its threads along x in 32 bits).  Those
// from n on have nothing to do.
inline dim3 wide_grid(uint64_t n) { return dim3(fp8_grid_x((uint32_t)n), fp8_grid_y((uint32_t)n)); }

// Division of numbers below 2^31 by a number that the host knows: n m / 2^shift with m = ceil(2^shift / d),
// shift = 31 + log2 d rounded up, is exact (m d exceeds 2^shift by less than d <= 2^(shift - 31)).
struct Divisor {
    uint32_t m, shift;
};
inline Divisor divisor(uint32_t d) {
    uint32_t shift = 31;
    while (((uint64_t)1 << (shift - 31)) < d) ++shift;
    return {(uint32_t)((((uint64_t)1 << shift) + d - 1) / d), shift};
}
#if defined(__HIPCC__)
__device__ inline int divide(int n, const Divisor& d) { return (int)((uint64_t)(uint32_t)n * d.m >> d.shift); }
#endif

// A packed tensor [tokens, heads, d]; strides in bytes.
struct QkRows {
    uint64_t p;
    int64_t  token, head;
};

// The pools and the table of a cache, and the step's lengths.
struct KvpPages {
    uint64_t       k, v;
    const int32_t* table;
    const int32_t* lens;
    const int32_t* tok0;          // null: sequence s has token s
    int64_t        table_stride;  // entries
    int64_t        page_stride;   // bytes
    int32_t        pages, page, columns, n_seq, kv_heads;
    int32_t        capacity;      // columns * page
    Divisor        by_page;
};

// ---- norm and rotation, with or without an append ----
// The rows of a token: `heads` of q, kv_heads of k and, with an append, as many of v.
struct QkParams {
    QkRows         q, k, v, q_out, k_out;  // (an append: k_out is the pages)
    const double*  freqs;
    const void*    wq;
    const void*    wk;
    const int32_t* pos;                    // null: the row number on every axis (append)
    int64_t        tokens;
    int32_t        heads, kv_heads, d, rot, axes;
    int32_t        tokens_wg;              // tokens of a workgroup, kQkTokens at most
    float          eps, w_add, inv_d;
    Divisor        by_rows;                // rows of a token
    bool           norm, pairs, w_f32;
    KvpPages       pages;
};
constexpr int kQkTokens = 8;
hipError_t launch_qk(const QkParams& p, bool f32, bool append, hipStream_t stream);

// ---- attend ----
// A segment is a KV head and `tile` query rows of a sequence (row r: token r / G, query head
// h G + r % G).  Its rows of the cache are cut into units of 32.  Either every segment is cut into even
// parts, a workgroup each, or the units of all segments in a row, each segment with `begin` more
// before it for what a segment costs, are dealt out in equal runs (tiles of 128: the units that each tile sees).  A workgroup has at most two segments that it
// shares with others, whose parts lie in its two slots of the workspace.
constexpr int kKvpUnit = 32;
struct KvpAttendParams {
    QkRows   q;
    void*    o;
    float*   lse;      // may be null
    float*   part_o;   // [2 wgs][tile][d], means
    float*   part_ml;  // [2 wgs][tile][2]: m (log2 units), sum
    uint64_t* meta;    // [tokens, heads]: first workgroup, parts, row of the segment
    int64_t  tokens;
    int32_t  heads, d, window;
    uint32_t wgs;
    int32_t  tile;     // query rows of a segment: 16, 32 or 128
    int32_t  begin;    // units that the beginning of a segment counts for
    int32_t  whole;    // segments are not cut, and there is no second launch
    float    scale_log2;  // not zero, so that scores that are masked by an infinity stay so
    Divisor  by_group, by_kv_heads;  // heads / kv_heads, kv_heads
    KvpPages pages;
};
hipError_t launch_kvp_attend(const KvpAttendParams& p, hipStream_t stream);

}  // namespace cap
