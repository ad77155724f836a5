// Blocks of a block-scaled FP8 KV cache for sparse attention on gfx950.
//
// A block's score for a token and KV head is the highest value that the product
// of a key within the block's bounds with any query of the head's group can have,
//   max_g sum_c max(q_gc lo_c, q_gc hi_c) * scale_k .
// With 2^a and 2^b the powers of two of a row's smallest (but zero) and largest values,
// the products with codes are multiples of 2^(a - 16) and 256 of them sum to less than
// 2^(b + 18): while the row spans less than 2^19 their sums are exact in 64 bits, in any
// order, and the choice does not depend on how a kernel adds.  A score that is NaN counts as
// infinite, as attention over the block gives NaN.
//
// Two launches.  Scores: q+ . hi + q- . lo (q+ and q- the positive and the negative part
// of q) on 64-bit matrix instructions, 16 query heads against 16 blocks to a workgroup,
// a quarter of the channels to a wave; written as ordered 64-bit keys.  Choice: one
// workgroup for each token and KV head finds the n_sel-th highest key by histograms of
// eight bits, from the highest bit in which the keys differ (above it every key would
// count into one bin), and writes the blocks in ascending order.  Blocks that a token
// has to have carry the highest key, those behind it the lowest.
// Both are bound by latency (16385 rows, 4 KV heads of 256 channels, one token: 5.0 us and 5.5;
// up to 131072 rows, 13 tokens: 10.6 and 9.7; with each digit found by the workgroup together
// instead of by every wave for itself, four barriers more to a digit, the choice took 6.2 and 10.9).
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "kvb_device.h"

namespace cap {
namespace {

using dev::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef double f64x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kKeysLds = 4096;    // keys that LDS holds
constexpr uint64_t kMust = ~0ull, kNever = 0;

__device__ inline uint64_t order_key(double x) {
    if (x != x) x = __builtin_inf();
    const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);  // one zero of the two
    return u >> 63 ? ~u : u | 1ull << 63;
}

template <int D, int N>
__global__ __launch_bounds__(kThreads) void score_kernel(const KvbSelectTable<N> p) {
    constexpr int kSteps = D / 16;  // channels of a lane: D / 4 to a wave, a quarter of them to a lane group
    __shared__ double part_s[4][4][64];
    __shared__ double best_s[4][16];
    const uint32_t block = kvb_block();
    if (block >= p.wgs) return;
    const KvbSelectSeq& s = p.seq[KVB_SEQ_OF(p, first_wg, block)];
    const uint32_t nb = (uint32_t)((s.n + kKvbBlock - 1) / kKvbBlock);
    const uint32_t parts = (nb + kKvbScoreBlocks - 1) / kKvbScoreBlocks;
    const uint32_t w = block - s.first_wg, pair = w / parts;
    const int h = (int)(pair % (uint32_t)p.kv_heads);
    const int64_t t = pair / (uint32_t)p.kv_heads;
    const uint32_t mine = (uint32_t)((s.n - s.T + t) / kKvbBlock);  // the token's own block
    const uint32_t b0 = (w - pair * parts) * kKvbScoreBlocks;
    const int tid = (int)threadIdx.x, lane = tid & 63, li = lane & 15, wave = tid >> 6;
    const int c0 = (wave * 4 + (lane >> 4)) * kSteps;  // the lane's channels, in both operands
    const int G = p.heads / p.kv_heads;

    // blocks past the last repeat it
    const uint32_t b = b0 + (uint32_t)li < nb ? b0 + (uint32_t)li : nb - 1;
    const global_ptr<uint8_t> lo = (global_ptr<uint8_t>)s.bounds + ((int64_t)b * 2 * p.kv_heads + h) * D + c0;
    uint32_t low[kSteps / 4], high[kSteps / 4];
    #pragma unroll
    for (int i = 0; i < kSteps / 4; ++i) {
        low[i] = *(global_ptr<uint32_t>)(lo + 4 * i);
        high[i] = *(global_ptr<uint32_t>)(lo + (int64_t)p.kv_heads * D + 4 * i);
    }
    double best = -__builtin_inf();
    bool nan = false;
    for (int g0 = 0; g0 < G; g0 += 16) {
        const int head = g0 + li < G ? g0 + li : G - 1;  // heads past the last repeat it
        const uint8_t* q = static_cast<const uint8_t*>(p.q) + (s.t0 + t) * p.q_stride + (((int64_t)h * G + head) * D + c0) * 2;
        uint32_t qs[kSteps / 2];
        #pragma unroll
        for (int i = 0; i < kSteps / 4; ++i) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(q + 8 * i);
            qs[2 * i] = x[0];
            qs[2 * i + 1] = x[1];
        }
        f64x4 acc = {0.0, 0.0, 0.0, 0.0};
        #pragma unroll
        for (int c = 0; c < kSteps; c += 2) {
            const f32x2 l = c & 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)low[c / 4], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)low[c / 4], false);
            const f32x2 u = c & 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)high[c / 4], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)high[c / 4], false);
            #pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float x = __builtin_bit_cast(float, e ? qs[c / 2] & 0xFFFF0000u : qs[c / 2] << 16);
                // (a NaN goes into both parts)
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(x < 0.0f ? 0.0f : x), (double)u[e], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)(x > 0.0f ? 0.0f : x), (double)l[e], acc, 0, 0, 0);
            }
        }
        if (g0) __syncthreads();
        #pragma unroll
        for (int r = 0; r < 4; ++r) part_s[wave][r][lane] = acc[r];
        __syncthreads();
        // accumulator r of all waves: some heads of block lane % 16; wave r sums it
        const double sum = (part_s[0][wave][lane] + part_s[1][wave][lane]) + (part_s[2][wave][lane] + part_s[3][wave][lane]);
        nan |= sum != sum;
        best = sum > best ? sum : best;
    }
    if (nan) best = __builtin_inf();
    #pragma unroll
    for (int o = 16; o < 64; o <<= 1) {
        const double x = __shfl_xor(best, o);
        best = x > best ? x : best;
    }
    if (lane < 16) best_s[wave][li] = best;
    __syncthreads();
    if (tid < 16 && b0 + (uint32_t)tid < nb) {
        #pragma unroll
        for (int i = 0; i < 4; ++i) best = best_s[i][tid] > best ? best_s[i][tid] : best;
        const float scale = ((global_ptr<float>)s.scales)[(int64_t)b * 2 * p.kv_heads + h];
        uint64_t key = order_key(best * (double)scale);
        if (b < (uint32_t)p.first || b + (uint32_t)p.last > mine) key = kMust;
        if (b > mine) key = kNever;
        p.keys[s.keys + pair * (uint64_t)nb + b] = key;
    }
}

template <int N>
__global__ __launch_bounds__(kThreads) void pick_kernel(const KvbSelectTable<N> p) {
    __shared__ uint64_t key_s[kKeysLds];
    __shared__ uint64_t range_s[kThreads / 64][2];
    __shared__ uint32_t waves[kThreads / 64];
    __shared__ uint64_t sums_s[kThreads / 64];
    __shared__ __attribute__((aligned(16))) uint32_t bins[8][256];  // a histogram for each digit
    static_assert(kThreads == 256, "a bin for each thread");
    const uint32_t block = kvb_block();
    if (block >= (uint32_t)(p.tokens * p.kv_heads)) return;
    const int64_t tok = block / (uint32_t)p.kv_heads;
    const int h = (int)(block - tok * p.kv_heads);
    const KvbSelectSeq& s = p.seq[KVB_SEQ_OF(p, t0, tok)];
    const int64_t t = tok - s.t0;
    const uint32_t nb = (uint32_t)((s.n + kKvbBlock - 1) / kKvbBlock);
    const uint32_t count = (uint32_t)((s.n - s.T + t) / kKvbBlock) + 1;  // blocks that the token sees some of
    const uint64_t* keys = p.keys + s.keys + (t * p.kv_heads + h) * (uint64_t)nb;
    int32_t* out = p.idx + (int64_t)block * p.n_sel;
    const uint32_t n_sel = (uint32_t)p.n_sel, tid = threadIdx.x;
    if (count <= n_sel) {
        for (uint32_t i = tid; i < n_sel; i += kThreads) out[i] = i < count ? (int32_t)i : -1;
        return;
    }
    const bool in_lds = count <= kKeysLds;
    #pragma unroll
    for (int i = 0; i < 8; ++i) bins[i][tid] = 0;
    // the highest and lowest key of those that the token need not have, and how many it has to
    uint64_t low = ~0ull, high = 0;
    uint32_t must = 0;
    constexpr int kBatch = 8;  // loads in flight
    for (uint32_t i0 = tid; i0 < count; i0 += kBatch * kThreads) {
        uint64_t k[kBatch];
        #pragma unroll
        for (int j = 0; j < kBatch; ++j) k[j] = keys[i0 + j * kThreads < count ? i0 + j * kThreads : i0];
        #pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint32_t i = i0 + j * kThreads;
            if (i >= count) continue;
            if (in_lds) key_s[i] = k[j];
            if (k[j] == kMust) {
                ++must;
            } else {
                low = k[j] < low ? k[j] : low;
                high = k[j] > high ? k[j] : high;
            }
        }
    }
    #pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint64_t l = __shfl_xor(low, o), h64 = __shfl_xor(high, o);
        low = l < low ? l : low;
        high = h64 > high ? h64 : high;
        must += __shfl_xor(must, o);
    }
    if ((tid & 63) == 0) {
        range_s[tid / 64][0] = low;
        range_s[tid / 64][1] = high;
        waves[tid / 64] = must;
    }
    __syncthreads();
    must = 0;
    #pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) {
        low = range_s[i][0] < low ? range_s[i][0] : low;
        high = range_s[i][1] > high ? range_s[i][1] : high;
        must += waves[i];
    }
    uint32_t need = n_sel - must;  // how many are still to be taken of the keys with the bits found so far
    int open = low == high ? 0 : 64 - __builtin_clzll(low ^ high);  // bits not found yet
    uint64_t prefix = open == 0 ? low : open == 64 ? 0 : low >> open << open;  // the bits found, the rest zero
    if (need == 0) {  // those it has to have, and no others
        prefix = kMust;
        need = ~0u;
        open = 0;
    }
    const int lane = (int)(tid & 63);
    for (int pass = 0; open > 0; ++pass) {
        const int width = open < 8 ? open : 8, shift = open - width;
        for (uint32_t i = tid; i < count; i += kThreads) {
            const uint64_t k = in_lds ? key_s[i] : keys[i];
            if (k != kMust && (open == 64 || (k ^ prefix) >> open == 0)) atomicAdd(&bins[pass][k >> shift & ((1u << width) - 1)], 1u);
        }
        __syncthreads();
        // the digit d with  #(digits > d) < need <= #(digits >= d), by each wave for itself: a
        // lane looks at four digits, from the highest down
        const u32x4 v = *reinterpret_cast<const u32x4*>(&bins[pass][252 - 4 * lane]);
        const uint32_t four = v[0] + v[1] + v[2] + v[3];
        uint32_t upto = four;  // inclusive sum over this lane and those before it
        #pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t x = __shfl_up(upto, o);
            if (lane >= o) upto += x;
        }
        uint32_t above = upto - four, digit = 255 - 4 * lane, size = v[3];
        const int at = __builtin_ctzll(__ballot(above < need && upto >= need));
        #pragma unroll
        for (int j = 2; j >= 0; --j)
            if (above + size < need) {
                above += size;
                size = v[j];
                --digit;
            }
        prefix |= (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)digit, at) << shift;
        need -= (uint32_t)__builtin_amdgcn_readlane((int)above, at);
        open = shift;
        if (need == (uint32_t)__builtin_amdgcn_readlane((int)size, at)) {  // all keys with these bits are taken
            need = ~0u;
            break;
        }
    }
    // ascending: every key above the bound, of those equal to it the first `need`; a thread
    // takes a run of blocks
    const uint32_t run = (count + kThreads - 1) / kThreads, i0 = tid * run < count ? tid * run : count;
    const uint32_t i1 = i0 + run < count ? i0 + run : count;
    uint32_t equal = 0, above = 0;
    for (uint32_t i = i0; i < i1; ++i) {
        const uint64_t k = in_lds ? key_s[i] : keys[i];
        equal += k == prefix;
        above += k > prefix;
    }
    const uint64_t both = (uint64_t)above << 32 | equal;
    uint64_t upto = both;  // the sums over the threads before this one, and it
    #pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t x = __shfl_up(upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 63) sums_s[tid / 64] = upto;
    __syncthreads();
    for (uint32_t i = 0; i < tid / 64; ++i) upto += sums_s[i];
    upto -= both;
    const uint32_t ties = (uint32_t)upto, taken = ties < need ? ties : need;
    uint32_t left = need - taken;  // ties that this thread may still take
    uint32_t at = (uint32_t)(upto >> 32) + taken;
    for (uint32_t i = i0; i < i1; ++i) {
        const uint64_t k = in_lds ? key_s[i] : keys[i];
        const bool tie = k == prefix && left > 0;
        if (tie) --left;
        if ((k > prefix || tie) && at < n_sel) out[at++] = (int32_t)i;
    }
}

template <int D>
hipError_t launch_score(const KvbSelectParams& p, hipStream_t stream) {
    return launch_kvb<KvbSelectTable>(reinterpret_cast<const void*>(&score_kernel<D, kKvbFew>),
                                      reinterpret_cast<const void*>(&score_kernel<D, KVB_MAX_SEQ>), kvb_grid(p.wgs), dim3(kThreads), p, stream);
}

}  // namespace

hipError_t launch_kvb_select(const KvbSelectParams& p, hipStream_t stream) {
    if (p.wgs == 0) return hipSuccess;
    const hipError_t e = p.d == 64 ? launch_score<64>(p, stream) : p.d == 128 ? launch_score<128>(p, stream) : launch_score<256>(p, stream);
    if (e != hipSuccess) return e;
    return launch_kvb<KvbSelectTable>(reinterpret_cast<const void*>(&pick_kernel<kKvbFew>), reinterpret_cast<const void*>(&pick_kernel<KVB_MAX_SEQ>),
                                      kvb_grid((uint32_t)(p.tokens * p.kv_heads)), dim3(kThreads), p, stream);
}

}  // namespace cap
