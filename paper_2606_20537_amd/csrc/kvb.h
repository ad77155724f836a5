// Internal interface of the block-scaled FP8 KV cache: the host checks and
// launch plans (kvb_host.cpp) and the kernels (kvb_append.hip, kvb_attend.hip,
// kvb_select.hip).  Not part of the public ABI.
#pragma once

#include "internal.h"

namespace cap {

constexpr int kKvbBlock = KVB_BLOCK;

// Parameters carry a table of sequences by value, of KVB_MAX_SEQ or of kKvbFew: a launch
// copies its arguments (4 KB of them 0.4 us of the host's 3.1).
// The table comes last, so that the short form is the beginning of the long one.
constexpr int kKvbFew = 4;

// A grid of workgroups of 256 (kvb_device.h: kvb_block): a launch counts its threads along x in
// 32 bits, which the scores of 46000 tokens on 8 KV heads pass.
inline dim3 kvb_grid(uint32_t wgs) { return dim3(fp8_grid_x(wgs), fp8_grid_y(wgs)); }

// ---- append ----
// Workgroup w works on sequence s with first_wg <= w < the next one's, on its
// block, KV head and side (K or V) number w - first_wg.
struct KvbAppendSeq {
    uint64_t k, v, scales, bounds, open;
    int64_t  n, t0;       // rows held with the new ones; first of the packed tokens
    int32_t  T;
    uint32_t first_wg;
};
template <int N>
struct KvbAppendTable {
    const void* k_new;
    const void* v_new;
    int64_t  k_stride, v_stride;  // bytes between tokens
    int32_t  n_seq, kv_heads, d;
    uint32_t wgs;
    KvbAppendSeq seq[N];
};
using KvbAppendParams = KvbAppendTable<KVB_MAX_SEQ>;
hipError_t launch_kvb_append(const KvbAppendParams& p, hipStream_t stream);

// ---- attend ----
// The query rows that share a KV head's K and V are taken in tiles of
// `tile` rows: row r of a sequence and KV head is token r / G, query head
// h G + r % G (G = heads / kv_heads); with a block list (sparse) the rows of
// one token.  The blocks of a tile are cut into nsplit runs of `per` blocks,
// each a workgroup; with more than one the runs leave (o, m, l) in slots of
// the workspace and a second launch joins them.
constexpr int kKvbListRun = 64;  // entries of a block list in one run
struct KvbAttendSeq {
    uint64_t k, v, scales;
    int64_t  n, t0;
    int32_t  T;
    uint32_t first_wg, first_slot;
    int32_t  per, nsplit;
    int32_t  pad;
};
template <int N>
struct KvbAttendTable {
    const void*    q;
    void*          o;
    float*         lse;        // may be null
    const int32_t* idx;        // null: every block
    float*         part_o;     // [slot][tile][d], not divided by l
    float*         part_ml;    // [slot][tile][2]: highest score (log2 units), sum
    int64_t        q_stride;   // bytes between tokens
    int64_t        tokens;
    int32_t        n_seq, heads, kv_heads, d, n_sel, tile;
    uint32_t       wgs, slots;
    float          scale_log2; // scale * log2(e)
    KvbAttendSeq   seq[N];
};
using KvbAttendParams = KvbAttendTable<KVB_MAX_SEQ>;

// Tiles of 16 rows (kvb_attend.hip) or of 128 (kvb_prefill.hip, no block list).
hipError_t launch_kvb_attend(const KvbAttendParams& p, hipStream_t stream);
hipError_t launch_kvb_prefill(const KvbAttendParams& p, hipStream_t stream);  // its first launch alone

// ---- select ----
struct KvbSelectSeq {
    uint64_t scales, bounds;
    int64_t  n, t0;
    int32_t  T;
    uint32_t first_wg;
    uint64_t keys;             // first sort key of the sequence in the workspace
};
template <int N>
struct KvbSelectTable {
    const void* q;
    int32_t*    idx;
    uint64_t*   keys;          // [token][kv head][blocks of the sequence]
    int64_t     q_stride, tokens;
    int32_t     n_seq, heads, kv_heads, d, n_sel, first, last;
    uint32_t    wgs;
    KvbSelectSeq seq[N];
};
using KvbSelectParams = KvbSelectTable<KVB_MAX_SEQ>;
// Blocks that one workgroup of the scoring launch takes.
constexpr int kKvbScoreBlocks = 16;
hipError_t launch_kvb_select(const KvbSelectParams& p, hipStream_t stream);

// Launch a kernel over a sequence table, in the form that its length asks for.
template <template <int> class Table>
inline hipError_t launch_kvb(const void* few, const void* many, dim3 grid, dim3 block, const Table<KVB_MAX_SEQ>& p,
                             hipStream_t stream) {
    void* args[] = {const_cast<Table<KVB_MAX_SEQ>*>(&p)};
    return hipLaunchKernel(p.n_seq <= kKvbFew ? few : many, grid, block, args, 0, stream);
}

}  // namespace cap
