// Device helpers shared by the kernels of the block-scaled FP8 KV cache.  Not
// part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include "kvb.h"

namespace cap {

template <typename T>
using global_ptr = const T __attribute__((address_space(1)))*;

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

}  // namespace cap
