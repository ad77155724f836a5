// Device helpers shared by the kernels of the block-scaled FP8 KV cache.  Not
// part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include "kvb.h"

namespace cap {

template <typename T>
using global_ptr = const T __attribute__((address_space(1)))*;

// A workgroup's number in a kvb_grid; those from the launch's count on have nothing to do.
__device__ inline uint32_t kvb_block() { return blockIdx.y * kFp8GridX + blockIdx.x; }

// The last sequence whose `field` (ascending) is at most x: lane i looks at
// sequence i, so that the table is read once, not once for each step of a search.
static_assert(KVB_MAX_SEQ <= 64, "a lane for each sequence");
template <class F>
__device__ inline int kvb_last(int n_seq, F&& upto) {
    if (n_seq == 1) return 0;
    const int lane = (int)(threadIdx.x & 63);
    return __builtin_popcountll(__ballot(lane < n_seq && upto(lane < n_seq ? lane : 0))) - 1;
}
#define KVB_SEQ_OF(p, field, x) ::cap::kvb_last((p).n_seq, [&](int i) { return (p).seq[i].field <= (x); })

// 0x80 in exactly the bytes of w that hold a NaN code (0x7F or 0xFF).
__device__ inline uint32_t nan_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// Rows of a sequence stay below 2^31 (the host's check): divided in 32 bits, as 64 take some
// 150 instructions, several times over before a workgroup's first load.
__device__ inline uint32_t row_div(int64_t row, int by) { return (uint32_t)row / (uint32_t)by; }
__device__ inline uint32_t row_mod(int64_t row, int by) { return (uint32_t)row % (uint32_t)by; }

// Blocks that the last row of a tile sees (rows row0 .. of a sequence's `total`; a token
// has G rows), and the runs they are cut into: later runs have nothing to do, and a tile
// with one run needs no join.
__device__ inline int tile_blocks(const KvbAttendSeq& s, int64_t row0, int tile, int64_t total, int G) {
    const int64_t last = row0 + tile < total ? row0 + tile - 1 : total - 1;
    return (int)((s.n - s.T + row_div(last, G)) / kKvbBlock) + 1;
}
__device__ inline int tile_runs(const KvbAttendSeq& s, int blocks) {
    const int runs = (blocks + s.per - 1) / s.per;
    return runs < s.nsplit ? runs : s.nsplit;
}

}  // namespace cap
