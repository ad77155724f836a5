// Norm of each head of q and k, rotation by position, and the append of the
// result to a paged bf16 cache, on gfx950.
//
//   y = x (mean x^2 + eps)^-1/2 (w_add + w)              over a head's d channels
//   a_i = sum over the axes of pos_axis freqs[axis][i]    i < rot / 2, in 64 bits
//   (y_a, y_b) -> (y_a cos a - y_b sin a, y_b cos a + y_a sin a)
//
// One pass: a row (one head of one token) lies in the registers of d / 16 lanes, each
// with two vectors of 8 channels that hold both channels of its pairs, so the only
// values that cross lanes are the sums of squares.  Sines and cosines are those
// of the token: a workgroup takes all heads of its tokens, computes each once and
// hands it round in LDS.  Everything between load and store is fp32, rounded once.
// The angle is taken in 64 bits and in turns, of which the whole ones go before it becomes
// two fp32 values: at position 2^20 the products alone would be off by 2^-4 in 32 bits.
//
// An append has the rows of v besides (copied), and k and v go to the row of the page
// that the table names; sequence, length and page of a token are found while its first rows are on their way.
//
// Bound by memory: 16384 tokens x 36 heads of 256 channels, 604 MB read and written, 114 us (5.3 TB/s, a
// copy of 1 GiB 5.2; without the arithmetic 111), in fp32, 1208 MB, 240 (5.0); the append of 40 heads, 671 MB, 127 us.  Stores are streamed
// (cached ones 123 us; 43 MB, which the last cache holds, 14 us against 11).  One row ahead of the one in work is
// on its way; with two the registers spill (132 us).
#include <hip/hip_runtime.h>

#include "kvp.h"

namespace cap {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kMostPairs = 256;  // rot <= 512

__device__ inline float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }

typedef char __attribute__((address_space(1)))* global_bytes;
typedef u32x4 __attribute__((address_space(1)))* global_u32x4;

// Eight channels as they lie in memory.  (Global addresses: an access by a generic one counts as one of LDS too, whose waits
// it would then hold up.)
template <bool F32>
struct Vec { u32x4 w[F32 ? 2 : 1]; };

template <bool F32>
__device__ inline Vec<F32> load8(global_bytes at) {
    Vec<F32> x;
    x.w[0] = *(const global_u32x4)at;
    if constexpr (F32) x.w[1] = *(const global_u32x4)(at + 16);
    return x;
}
template <bool F32>
__device__ inline void store8(global_bytes at, const Vec<F32>& x) {
    __builtin_nontemporal_store(x.w[0], (global_u32x4)at);
    if constexpr (F32) __builtin_nontemporal_store(x.w[1], (global_u32x4)(at + 16));
}
template <bool F32>
__device__ inline void widen(const Vec<F32>& x, float* f) {
    #pragma unroll
    for (int e = 0; e < 8; ++e)
        if constexpr (F32) f[e] = bits_f32(x.w[e / 4][e % 4]);
        else f[e] = bits_f32(e & 1 ? x.w[0][e / 2] & 0xFFFF0000u : x.w[0][e / 2] << 16);
}
// Rounded where values have changed (~0); else the bits that they came with, those of a NaN too.
template <bool F32>
__device__ inline Vec<F32> narrow(const float* f, uint32_t changed) {
    Vec<F32> x;
    #pragma unroll
    for (int e = 0; e < 8; e += 2) {
        if constexpr (F32) {
            x.w[e / 4][e % 4] = __builtin_bit_cast(uint32_t, f[e]);
            x.w[e / 4][e % 4 + 1] = __builtin_bit_cast(uint32_t, f[e + 1]);
        } else {
            const uint32_t rounded = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){f[e], f[e + 1]}, bf16x2));
            const uint32_t same = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, f[e + 1]), __builtin_bit_cast(uint32_t, f[e]), 0x07060302u);
            x.w[0][e / 2] = (rounded & changed) | (same & ~changed);
        }
    }
    return x;
}

// The factor of channel c.
__device__ inline float weight(const void* w, int c, const QkParams& p) {
    if (!w) return 1.0f;
    return p.w_add + (p.w_f32 ? static_cast<const float*>(w)[c] : bits_f32((uint32_t)static_cast<const uint16_t*>(w)[c] << 16));
}

// Sum over `lanes` (a power of two, 32 at most) neighbouring lanes, in all of them: neighbours, pairs, and mirrored
// quarters and halves of 16 lanes (whose values are equal by then) by cross-lane ALU operations.
template <int CTRL>
__device__ inline float moved(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ inline float sum_lanes(float x, int lanes) {
    if (lanes > 1) x += moved<0xB1>(x);   // quad_perm 1 0 3 2
    if (lanes > 2) x += moved<0x4E>(x);   // quad_perm 2 3 0 1
    if (lanes > 4) x += moved<0x141>(x);  // row_half_mirror
    if (lanes > 8) x += moved<0x140>(x);  // row_mirror
    if (lanes > 16) x += __shfl_xor(x, 16);
    return x;
}

// The sequence of packed token t: the last one that begins at or before it (-1: none).
// A wave looks at 64 of them at once.
__device__ inline int seq_of(const KvpPages& g, int t) {
    const int lane = (int)(threadIdx.x & 63);
    const int step = (g.n_seq + 63) / 64;  // 16 at most
    int s = -1;
    if (step > 1) {
        const int i = lane * step;
        const int n = __builtin_popcountll(__ballot(i < g.n_seq && g.tok0[i < g.n_seq ? i : 0] <= t));
        if (n == 0) return -1;
        s = (n - 1) * step;
    } else {
        s = 0;
    }
    const int i = s + lane;
    const bool here = lane < (step > 1 ? step : 64) && i < g.n_seq;
    return s + __builtin_popcountll(__ballot(here && g.tok0[here ? i : 0] <= t)) - 1;
}

template <bool F32, bool APPEND>
__global__ __launch_bounds__(kThreads, F32 ? 5 : 6) void rotate_kernel(const QkParams p) {
    constexpr int kSize = F32 ? 4 : 2;
    __shared__ __attribute__((aligned(16))) float cs_s[kQkTokens * kMostPairs * 2];  // cosine, sine
    __shared__ __attribute__((aligned(16))) float w_s[2][2 * kMostPairs];            // factors of q's channels and of k's
    __shared__ int64_t off_s[kQkTokens];  // bytes from a pool's begin to the token's row; -1: on no page; -2: of no sequence
    __shared__ int row_s[kQkTokens];      // its number
    const int tid = (int)threadIdx.x;
    const int64_t t0 = ((int64_t)blockIdx.y * kFp8GridX + blockIdx.x) * p.tokens_wg;
    if (t0 >= p.tokens) return;
    const int here = (int)(p.tokens - t0 < p.tokens_wg ? p.tokens - t0 : p.tokens_wg);
    const int half = p.rot / 2;

    // a lane's channels: 8 from `a` and 8 from `b`
    const int slots = p.d / 16;
    int lanes = 1;
    while (lanes < slots) lanes *= 2;
    const int slot = tid & (lanes - 1);
    const bool in = slot < slots;
    int a, b, first = -1;  // first: a's first pair; -1: not rotated (halves)
    if (p.pairs) {
        a = 8 * slot;
        b = p.d / 2 + 8 * slot;
    } else if (8 * slot < half) {
        a = first = 8 * slot;
        b = half + 8 * slot;
    } else {
        a = p.rot + 8 * slot - half;
        b = a + (p.d - p.rot) / 2;
    }
    // rows of the workgroup's tokens in order: q's heads, k's, and (append) v's
    const int of_q = p.heads, of_qk = p.heads + p.kv_heads, all = APPEND ? of_qk + p.kv_heads : of_qk;
    const int rows = here * all, per = kThreads / lanes;
    Vec<F32> va, vb;
    auto load_row = [&](int t, int head) {
        const QkRows& src = head < of_q ? p.q : head < of_qk ? p.k : p.v;
        const int h = head < of_q ? head : head < of_qk ? head - of_q : head - of_qk;
        const global_bytes from = (global_bytes)src.p + (t0 + t) * src.token + (int64_t)h * src.head;
        va = load8<F32>(from + a * kSize);
        vb = load8<F32>(from + b * kSize);
    };
    int r = tid / lanes, t = divide(r, p.by_rows), head = r - t * all;
    if (in && r < rows) load_row(t, head);  // on its way while angles and pages are found

    if (p.norm) {
        for (int c = tid; c < p.d; c += kThreads) {
            w_s[0][c] = weight(p.wq, c, p);
            w_s[1][c] = weight(p.wk, c, p);
        }
    }
    if constexpr (APPEND) {
        const KvpPages& g = p.pages;
        for (int i = tid >> 6; i < here; i += kThreads / 64) {
            const int token = (int)(t0 + i);
            int seq = -1, row = 0;
            if (g.tok0) {
                const int s = __builtin_amdgcn_readfirstlane(seq_of(g, token));
                if (s >= 0) {
                    const int end = g.tok0[s + 1];
                    row = (int)((int64_t)g.lens[s] - end + token);
                    if (token < end && row >= 0) seq = s;
                }
            } else if (token < g.n_seq) {
                row = g.lens[token] - 1;
                if (row >= 0) seq = token;
            }
            int64_t off = seq < 0 ? -2 : -1;
            if (seq >= 0 && row < g.capacity) {
                const int column = divide(row, g.by_page);
                const int page = g.table[(int64_t)seq * g.table_stride + column];
                if ((uint32_t)page < (uint32_t)g.pages)
                    off = (int64_t)page * g.page_stride + (int64_t)(row - column * g.page) * (g.kv_heads * p.d * 2);
            }
            if ((tid & 63) == 0) {
                off_s[i] = off;
                row_s[i] = row;
            }
        }
        __syncthreads();
    }
    // sines and cosines of the workgroup's tokens
    for (int i = tid; i < here * half; i += kThreads) {
        const int token = (int)((uint32_t)i / (uint32_t)half), pair = i - token * half;
        double turns = 0.0;
        for (int x = 0; x < p.axes; ++x) {
            const int at = APPEND && !p.pos ? row_s[token] : p.pos[(t0 + token) * p.axes + x];
            turns += (double)at * p.freqs[(int64_t)x * half + pair];
        }
        turns *= 0.15915494309189533577;  // 1 / (2 pi)
        turns -= __builtin_rint(turns);
        // what fp32 leaves of the angle turns the pair once more
        const float near = (float)turns, rest = 6.2831853f * (float)(turns - (double)near);
        float sine, cosine;
        sincospif(2.0f * near, &sine, &cosine);
        *reinterpret_cast<f32x2*>(&cs_s[2 * i]) = (f32x2){__builtin_fmaf(-rest, sine, cosine), __builtin_fmaf(rest, cosine, sine)};
    }
    __syncthreads();

    while (r < rows) {
        const int now_t = t, now_head = head;
        const Vec<F32> ua = va, ub = vb;
        r += per;
        for (head += per; head >= all; head -= all) ++t;
        if (in && r < rows) load_row(t, head);  // the next row

        global_bytes to;
        bool write = in;
        if (APPEND && now_head >= of_q) {
            const int h = now_head < of_qk ? now_head - of_q : now_head - of_qk;
            to = (global_bytes)(now_head < of_qk ? p.pages.k : p.pages.v) + off_s[now_t] + (int64_t)h * p.d * 2;
            write = in && off_s[now_t] >= 0;
        } else {
            const QkRows& dst = now_head < of_q ? p.q_out : p.k_out;
            const int h = now_head < of_q ? now_head : now_head - of_q;
            to = (global_bytes)dst.p + (t0 + now_t) * dst.token + (int64_t)h * dst.head;
            if (APPEND) write = in && off_s[now_t] != -2;
        }
        Vec<F32> oa = ua, ob = ub;
        if (now_head < of_qk) {  // (uniform over a row's lanes)
            float x[16];
            #pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 0.0f;
            if (in) {
                widen<F32>(ua, x);
                widen<F32>(ub, x + 8);
            }
            if (p.norm) {
                float sum = 0.0f;
                #pragma unroll
                for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
                sum = sum_lanes(sum, lanes);
                float eps = p.eps;
                if (!(sum < __builtin_inff())) {  // squares that overflow: the row in units of 2^70
                    sum = 0.0f;
                    #pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        x[e] *= 0x1p-70f;
                        sum = __builtin_fmaf(x[e], x[e], sum);
                    }
                    sum = sum_lanes(sum, lanes);
                    eps = 0.0f;
                }
                const float f = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, p.inv_d, eps));
                const float* w = w_s[now_head < of_q ? 0 : 1];
                #pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 four = *reinterpret_cast<const f32x4*>(&w[in ? (e < 8 ? a + e : b + e - 8) : 0]);
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) x[e + i] = x[e + i] * f * four[i];
                }
            }
            if (p.pairs) {
                #pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const int pair = ((e < 8 ? a + e : b + e - 8)) / 2;
                    if (in && pair < half) {
                        const f32x2 cs = *reinterpret_cast<const f32x2*>(&cs_s[2 * (now_t * half + pair)]);
                        const float y0 = x[e], y1 = x[e + 1];
                        x[e] = y0 * cs[0] - y1 * cs[1];
                        x[e + 1] = y1 * cs[0] + y0 * cs[1];
                    }
                }
            } else if (in && first >= 0) {
                #pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const f32x4 cs = *reinterpret_cast<const f32x4*>(&cs_s[2 * (now_t * half + first + e)]);
                    #pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float y0 = x[e + i], y1 = x[8 + e + i];
                        x[e + i] = y0 * cs[2 * i] - y1 * cs[2 * i + 1];
                        x[8 + e + i] = y1 * cs[2 * i] + y0 * cs[2 * i + 1];
                    }
                }
            }
            oa = narrow<F32>(x, p.norm || (p.pairs ? a < p.rot : first >= 0) ? ~0u : 0u);
            ob = narrow<F32>(x + 8, p.norm || (p.pairs ? b < p.rot : first >= 0) ? ~0u : 0u);
        }
        if (write) {
            store8<F32>(to + a * kSize, oa);
            store8<F32>(to + b * kSize, ob);
        }
    }
}

}  // namespace

hipError_t launch_qk(const QkParams& p, bool f32, bool append, hipStream_t stream) {
    const void* kernel = append ? reinterpret_cast<const void*>(&rotate_kernel<false, true>)
                         : f32  ? reinterpret_cast<const void*>(&rotate_kernel<true, false>)
                                : reinterpret_cast<const void*>(&rotate_kernel<false, false>);
    void* args[] = {const_cast<QkParams*>(&p)};
    return hipLaunchKernel(kernel, wide_grid((uint64_t)((p.tokens + p.tokens_wg - 1) / p.tokens_wg)), dim3(kThreads), args, 0, stream);
}

}  // namespace cap
