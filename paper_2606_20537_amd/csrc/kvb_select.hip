// Blocks of a block-scaled FP8 KV cache for sparse attention on gfx950.
//
// A block's score for a token and KV head is the highest value that the product
// of a key within the block's bounds with any query of the head's group can have,
//   max_g sum_c max(q_gc lo_c, q_gc hi_c) * scale_k .
// Products of bf16 and E4M3 values have 12 bits, so in 64 bits their sums are
// exact in any order (as long as a row's values span less than 2^30), and the
// choice does not depend on how a kernel adds.  A score that is NaN counts as
// infinite, as attention over the block gives NaN.
//
// Two launches: scores as ordered 64-bit keys, 32 blocks to a workgroup, eight
// threads to a block; then one workgroup for each token and KV head finds the
// n_sel-th highest key by its bytes from the top (a histogram of 256 in LDS for
// each) and writes the blocks in ascending order.  Blocks that a token has to
// have carry the highest key, those behind it the lowest.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "kvb_device.h"

namespace cap {
namespace {

using dev::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kHeads = 8;         // query heads that LDS holds at a time
constexpr int kKeysLds = 4096;    // keys that LDS holds
constexpr uint64_t kMust = ~0ull, kNever = 0;

__device__ inline uint64_t order_key(double x) {
    if (x != x) x = __builtin_inf();
    const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);  // one zero of the two
    return u >> 63 ? ~u : u | 1ull << 63;
}

template <int D>
__global__ __launch_bounds__(kThreads) void score_kernel(const KvbSelectParams p) {
    constexpr int kPer = D / 8;  // channels of a thread
    __shared__ float q_s[kHeads][D];
    const KvbSelectSeq& s = p.seq[KVB_SEQ_OF(p, first_wg, blockIdx.x)];
    const uint32_t nb = (uint32_t)((s.n + kKvbBlock - 1) / kKvbBlock);
    const uint32_t parts = (nb + kKvbScoreBlocks - 1) / kKvbScoreBlocks;
    const uint32_t w = blockIdx.x - s.first_wg, pair = w / parts;
    const int h = (int)(pair % (uint32_t)p.kv_heads);
    const int64_t t = pair / (uint32_t)p.kv_heads;
    const uint32_t mine = (uint32_t)((s.n - s.T + t) / kKvbBlock);  // the token's own block
    const int tid = (int)threadIdx.x, part = tid & 7, c0 = part * kPer;
    const uint32_t b = (w - pair * parts) * kKvbScoreBlocks + (uint32_t)tid / 8;
    const int G = p.heads / p.kv_heads;

    const uint8_t* q = static_cast<const uint8_t*>(p.q) + (s.t0 + t) * p.q_stride + (int64_t)h * G * D * 2;
    float lof[kPer], hif[kPer];
    {
        const uint8_t* base = reinterpret_cast<const uint8_t*>(s.bounds) + ((int64_t)(b < nb ? b : nb - 1) * 2 * p.kv_heads + h) * D + c0;
        const uint8_t* top = base + (int64_t)p.kv_heads * D;
        #pragma unroll
        for (int i = 0; i < kPer / 8; ++i) {
            const u32x2 a = *reinterpret_cast<const u32x2*>(base + 8 * i), z = *reinterpret_cast<const u32x2*>(top + 8 * i);
            #pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x2 a0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)a[k], false), a1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)a[k], true);
                const f32x2 z0 = __builtin_amdgcn_cvt_pk_f32_fp8((int)z[k], false), z1 = __builtin_amdgcn_cvt_pk_f32_fp8((int)z[k], true);
                #pragma unroll
                for (int e = 0; e < 2; ++e) {
                    lof[8 * i + 4 * k + e] = a0[e];
                    lof[8 * i + 4 * k + 2 + e] = a1[e];
                    hif[8 * i + 4 * k + e] = z0[e];
                    hif[8 * i + 4 * k + 2 + e] = z1[e];
                }
            }
        }
    }
    double best = -__builtin_inf();
    bool nan = false;
    for (int g0 = 0; g0 < G; g0 += kHeads) {
        const int heads = G - g0 < kHeads ? G - g0 : kHeads;
        __syncthreads();
        for (int i = tid; i < heads * D / 2; i += kThreads) {
            const uint32_t u = *reinterpret_cast<const uint32_t*>(q + ((int64_t)g0 * D + 2 * i) * 2);
            q_s[2 * i / D][2 * i % D] = __builtin_bit_cast(float, u << 16);
            q_s[2 * i / D][2 * i % D + 1] = __builtin_bit_cast(float, u & 0xFFFF0000u);
        }
        __syncthreads();
        for (int g = 0; g < heads; ++g) {
            double sum = 0.0;
            #pragma unroll
            for (int c = 0; c < kPer; ++c) {
                const float x = q_s[g][c0 + c];
                sum = __builtin_fma((double)x, (double)(x < 0.0f ? lof[c] : hif[c]), sum);
            }
            #pragma unroll
            for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor(sum, o);
            nan |= sum != sum;
            best = sum > best ? sum : best;
        }
    }
    if (part == 0 && b < nb) {
        const float scale = reinterpret_cast<const float*>(s.scales)[(int64_t)b * 2 * p.kv_heads + h];
        uint64_t key = order_key(nan ? __builtin_inf() : best * (double)scale);
        if (b < (uint32_t)p.first || b + (uint32_t)p.last > mine) key = kMust;
        if (b > mine) key = kNever;
        p.keys[s.keys + pair * (uint64_t)nb + b] = key;
    }
}

__global__ __launch_bounds__(kThreads) void pick_kernel(const KvbSelectParams p) {
    __shared__ uint64_t key_s[kKeysLds];
    __shared__ uint32_t bins[256], found[2], waves[kThreads / 64];
    const int64_t tok = blockIdx.x / (uint32_t)p.kv_heads;
    const int h = (int)(blockIdx.x - tok * p.kv_heads);
    const KvbSelectSeq& s = p.seq[KVB_SEQ_OF(p, t0, tok)];
    const int64_t t = tok - s.t0;
    const uint32_t nb = (uint32_t)((s.n + kKvbBlock - 1) / kKvbBlock);
    const uint32_t count = (uint32_t)((s.n - s.T + t) / kKvbBlock) + 1;  // blocks that the token sees some of
    const uint64_t* keys = p.keys + s.keys + (t * p.kv_heads + h) * (uint64_t)nb;
    int32_t* out = p.idx + (int64_t)blockIdx.x * p.n_sel;
    const uint32_t n_sel = (uint32_t)p.n_sel, tid = threadIdx.x;
    if (count <= n_sel) {
        for (uint32_t i = tid; i < n_sel; i += kThreads) out[i] = i < count ? (int32_t)i : -1;
        return;
    }
    const bool in_lds = count <= kKeysLds;
    if (in_lds)
        for (uint32_t i = tid; i < count; i += kThreads) key_s[i] = keys[i];
    uint64_t prefix = 0;     // the bytes found so far, the rest zero
    uint32_t need = n_sel;   // how many are still to be taken of the keys with these bytes
    for (int shift = 56; shift >= 0; shift -= 8) {
        bins[tid] = 0;
        __syncthreads();
        for (uint32_t i = tid; i < count; i += kThreads) {
            const uint64_t k = in_lds ? key_s[i] : keys[i];
            if (shift == 56 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&bins[k >> shift & 255], 1u);
        }
        __syncthreads();
        // the byte d with  #(bytes > d) < need <= #(bytes >= d): thread tid looks at d = 255 - tid
        const uint32_t mine = bins[255 - tid];
        uint32_t upto = mine;  // inclusive sum over this thread and those before it
        #pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t v = __shfl_up(upto, o);
            if ((int)(tid & 63) >= o) upto += v;
        }
        if ((tid & 63) == 63) waves[tid / 64] = upto;
        __syncthreads();
        for (uint32_t i = 0; i < tid / 64; ++i) upto += waves[i];
        if (upto >= need && upto - mine < need) {
            found[0] = 255 - tid;
            found[1] = need - (upto - mine);
        }
        __syncthreads();
        prefix |= (uint64_t)found[0] << shift;
        need = found[1];
        if (need == bins[found[0]]) {  // all keys with these bytes are taken
            need = ~0u;
            break;
        }
        __syncthreads();  // the bins are read before they are cleared
    }
    __syncthreads();
    // ascending: every key above the bound, of those equal to it the first `need`
    uint32_t done = 0, ties = 0;
    for (uint32_t i0 = 0; i0 < count; i0 += kThreads) {
        const uint32_t i = i0 + tid;
        const uint64_t k = i < count ? (in_lds ? key_s[i] : keys[i]) : 0;
        const bool equal = i < count && k == prefix;
        const uint64_t eq = __ballot(equal);
        const uint32_t below = __builtin_amdgcn_mbcnt_hi((uint32_t)(eq >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)eq, 0));
        if ((tid & 63) == 0) waves[tid / 64] = (uint32_t)__builtin_popcountll(eq);
        __syncthreads();
        uint32_t tie = ties + below, all = 0;
        for (uint32_t j = 0; j < kThreads / 64; ++j) {
            if (j < tid / 64) tie += waves[j];
            all += waves[j];
        }
        ties += all;
        const bool take = i < count && (k > prefix || (equal && tie < need));
        const uint64_t tk = __ballot(take);
        const uint32_t before = __builtin_amdgcn_mbcnt_hi((uint32_t)(tk >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)tk, 0));
        __syncthreads();
        if ((tid & 63) == 0) waves[tid / 64] = (uint32_t)__builtin_popcountll(tk);
        __syncthreads();
        uint32_t at = done + before;
        for (uint32_t j = 0; j < kThreads / 64; ++j) {
            if (j < tid / 64) at += waves[j];
            done += waves[j];
        }
        if (take && at < n_sel) out[at] = (int32_t)i;
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_kvb_select(const KvbSelectParams& p, hipStream_t stream) {
    if (p.wgs == 0) return hipSuccess;
    const void* fn = p.d == 64    ? reinterpret_cast<const void*>(&score_kernel<64>)
                     : p.d == 128 ? reinterpret_cast<const void*>(&score_kernel<128>)
                                  : reinterpret_cast<const void*>(&score_kernel<256>);
    const hipError_t e = launch_kernel(fn, dim3(p.wgs), dim3(kThreads), p, stream);
    if (e != hipSuccess) return e;
    return launch_kernel(reinterpret_cast<const void*>(&pick_kernel), dim3((uint32_t)(p.tokens * p.kv_heads)), dim3(kThreads), p,
                         stream);
}

}  // namespace cap
