// Causal attention of many query rows over a block-scaled FP8 KV cache on gfx950
// (the formulas and the sharing of K and V by a group's heads: kvb_attend.hip).
//
// A workgroup of four waves takes 128 query rows of a KV head, 32 to a wave, and
// walks the blocks; K and V codes of a block go through LDS, two buffers, one
// barrier a block.  Both products run on 32x32x64 FP8 tiles straight from the
// codes, with the power-of-two scales as the instruction's scale operands:
//  * S^T = K Q^T: a bf16 query row as hi + lo / 16 of E4M3 (kvb_attend.hip); the
//    scales of K and of lo cost nothing.
//  * O^T = V^T P^T: the weights of a block are taken against the block's own
//    highest score, rounded up to an integer c in log2 units, w = 2^(x - c + 8) in
//    (0, 256], and split like Q: w = hi + lo / 16 with a relative error of 2^-8 at
//    most, that of bf16, or 2^-22 of the block's largest weight where that is more.
//    2^(c - m), m the running maximum of the c, is the instruction's scale of a
//    row: an exact power of two, as are all corrections of O and l.
// Against bf16 operands that is the same matrix time (FP8 runs at twice the rate),
// half the LDS traffic and no conversion of K and V.
//
// A lane has one query row in both products and S^T's accumulators are P^T's
// operand: byte 4 j + i of lane half h is key 8 j + 4 h + i.  V's operand has its
// keys in the same order, read with the transposing 8-byte LDS read.  Rows in LDS
// are permuted in 16-byte units so that both reads are free of bank conflicts.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "kvb.h"

namespace cap {
namespace {

using dev::rsrc_t;
using dev::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr float kNegInf = -__builtin_inff();
constexpr float kLn2 = 0.6931471805599453f;

__device__ inline float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ inline uint32_t f32_bits(float f) { return __builtin_bit_cast(uint32_t, f); }
__device__ inline float pair_max(float x) { return __builtin_fmaxf(x, __shfl_xor(x, 32)); }

// 0x80 in exactly the bytes of w that hold a NaN code (0x7F or 0xFF).
__device__ inline uint32_t nan_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// Four values to four E4M3 codes, and their remainders times 16 to four more.
__device__ inline void split4(const float* y, int& hi, int& lo) {
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32((y[2] - b[0]) * 16.0f, (y[3] - b[1]) * 16.0f,
                                         __builtin_amdgcn_cvt_pk_fp8_f32((y[0] - a[0]) * 16.0f, (y[1] - a[1]) * 16.0f, 0, false), true);
}

__device__ inline f32x16 mma(const i32x8& a, const i32x8& b, const f32x16& c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

// Where the 16-byte unit `u` of row `key` lies in its row: the reads of K take
// one unit of eight neighbouring rows at a time, those of V of rows i and 8 + i
// (i = 0..3 or 4..7).
template <int D>
__device__ inline int swizzle_k(int key) { return D == 64 ? key >> 1 & 3 : key & 7; }
template <int D>
__device__ inline int swizzle_v(int key) {
    return D == 64 ? (key >> 1 & 1) | (key >> 3 & 1) << 1 : (key & 3) | (key >> 3 & 1) << 2;
}

template <int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void prefill_kernel(const KvbAttendParams p) {
    constexpr int NJ = D / 64, NT = D / 32, kUnits = D / 16, kRows = kThreads / kUnits, kLoads = kKvbBlock / kRows;
    __shared__ __attribute__((aligned(1024))) uint8_t k_s[2][kKvbBlock * D];
    __shared__ __attribute__((aligned(1024))) uint8_t v_s[2][kKvbBlock * D];
    __shared__ int nan_s[2];

    int lo = 0, hi = p.n_seq - 1;  // last s with first_wg <= blockIdx.x
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.seq[mid].first_wg <= blockIdx.x) lo = mid; else hi = mid - 1;
    }
    const KvbAttendSeq& s = p.seq[__builtin_amdgcn_readfirstlane(lo)];
    const uint32_t w = blockIdx.x - s.first_wg;
    const int G = p.heads / p.kv_heads;
    const uint32_t item = w / (uint32_t)s.nsplit;
    const int split = (int)(w - item * (uint32_t)s.nsplit);
    const int h = (int)(item % (uint32_t)p.kv_heads);
    const int64_t total = (int64_t)s.T * G, tiles = (total + 127) / 128;
    const int64_t tile = tiles - 1 - item / (uint32_t)p.kv_heads;  // the longest first
    const int tid = (int)threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row0 = tile * 128, wrow0 = row0 + wave * 32, last = total - 1;
    const int64_t row = wrow0 + (lane & 31) < last ? wrow0 + (lane & 31) : last;  // rows past the last repeat it
    const int64_t before = s.n - s.T, token = row / G, pos = before + token;     // the last key that the row sees
    // the wave's first and last position, and the tile's
    const int64_t wpos0 = before + (wrow0 < last ? wrow0 : last) / G, wpos1 = before + (wrow0 + 31 < last ? wrow0 + 31 : last) / G;
    const int64_t tpos0 = before + row0 / G, tpos1 = before + (row0 + 127 < last ? row0 + 127 : last) / G;

    i32x8 qh[NJ], ql[NJ];
    float f;  // from the products to log2 units
    {
        const uint8_t* src = static_cast<const uint8_t*>(p.q) + (s.t0 + token) * p.q_stride + ((int64_t)h * G + row % G) * D * 2;
        u32x4 x[NJ][4];
        float amax = 0.0f;
        #pragma unroll
        for (int j = 0; j < NJ; ++j)
            #pragma unroll
            for (int c = 0; c < 4; ++c) {
                x[j][c] = *reinterpret_cast<const u32x4*>(src + (64 * j + 32 * (c / 2) + 16 * half + 8 * (c % 2)) * 2);
                #pragma unroll
                for (int k = 0; k < 4; ++k)
                    amax = __builtin_fmaxf(amax, __builtin_fmaxf(__builtin_fabsf(bits_f32(x[j][c][k] << 16)),
                                                                 __builtin_fabsf(bits_f32(x[j][c][k] & 0xFFFF0000u))));
            }
        amax = pair_max(amax);
        int e = (int)(f32_bits(amax) >> 23) - 127 - 7;  // amax 2^-e in [128, 256)
        e = e < -100 ? -100 : e;
        const float mul = bits_f32((uint32_t)(127 - e) << 23);  // an infinity stays one, and becomes NaN
        f = bits_f32((uint32_t)(127 + e) << 23) * p.scale_log2;
        #pragma unroll
        for (int j = 0; j < NJ; ++j)
            #pragma unroll
            for (int c = 0; c < 8; ++c) {
                float y[4];
                #pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t u = x[j][c / 2][2 * (c % 2) + k];
                    y[2 * k] = bits_f32(u << 16) * mul;
                    y[2 * k + 1] = bits_f32(u & 0xFFFF0000u) * mul;
                }
                int a, b;
                split4(y, a, b);
                qh[j][c] = a;
                ql[j][c] = b;
            }
    }

    const int rowb = p.kv_heads * D;
    const uint8_t* kb = reinterpret_cast<const uint8_t*>(s.k);
    const uint8_t* vb = reinterpret_cast<const uint8_t*>(s.v);
    const float* sc = reinterpret_cast<const float*>(s.scales);
    const int begin = split * s.per;
    const int nblk = (int)(tpos1 / kKvbBlock) + 1, end = begin + s.per < nblk ? begin + s.per : nblk;

    // staging: thread tid moves unit tid % kUnits of rows tid / kUnits + i kRows
    const int srow = tid / kUnits, sunit = tid % kUnits;
    const int svoff = srow * rowb + h * D + 16 * sunit;
    u32x4 ks[kLoads], vs[kLoads];
    auto fetch = [&](int b) {
        const rsrc_t rk = dev::make_rsrc_u32(kb + (int64_t)b * kKvbBlock * rowb, (uint32_t)kKvbBlock * rowb);
        const rsrc_t rv = dev::make_rsrc_u32(vb + (int64_t)b * kKvbBlock * rowb, (uint32_t)kKvbBlock * rowb);
        #pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            ks[i] = __builtin_amdgcn_raw_buffer_load_b128(rk, svoff, i * kRows * rowb, 0);
            vs[i] = __builtin_amdgcn_raw_buffer_load_b128(rv, svoff, i * kRows * rowb, 0);
        }
    };
    auto stage = [&](int b, int buf) {
        // Where some row does not see every key, NaN codes of V go (a weight of zero
        // would make them NaN), and are put back after the product.
        if ((int64_t)b * kKvbBlock + kKvbBlock - 1 > tpos0) {
            bool seen = false;
            #pragma unroll
            for (int i = 0; i < kLoads; ++i)
                #pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t bad = nan_bytes(vs[i][k]);
                    seen |= bad != 0 && (int64_t)b * kKvbBlock + srow + i * kRows < s.n;
                    vs[i][k] &= ~(bad | (bad - (bad >> 7)));
                }
            if (seen) nan_s[buf] = b;
        }
        #pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int key = srow + i * kRows;
            *reinterpret_cast<u32x4*>(&k_s[buf][key * D + 16 * (sunit ^ swizzle_k<D>(key))]) = ks[i];
            *reinterpret_cast<u32x4*>(&v_s[buf][key * D + 16 * (sunit ^ swizzle_v<D>(key))]) = vs[i];
        }
    };

    // addresses of a lane's reads; units and rows come in by xor and offset
    const int kaddr = (lane & 31) * D + 16 * (half ^ swizzle_k<D>(lane & 31));
    const int vkey = 4 * half + ((lane & 15) >> 1 & 3) + 8 * ((lane & 15) >> 3);
    const int vaddr = vkey * D + 16 * ((lane >> 4 & 1) ^ swizzle_v<D>(vkey)) + 8 * (lane & 1);

    f32x16 acc[NT];
    #pragma unroll
    for (int c = 0; c < NT; ++c)
        #pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] = 0.0f;
    float m = kNegInf, l = 0.0f;

    if (tid < 2) nan_s[tid] = -1;
    if (begin < end) fetch(begin);
    __syncthreads();
    if (begin < end) stage(begin, 0);
    for (int b = begin; b < end; ++b) {
        const int buf = (b - begin) & 1;
        __syncthreads();
        if (b + 1 < end) fetch(b + 1);
        const int64_t r0 = (int64_t)b * kKvbBlock;
        if (r0 <= wpos1) {
            const int k_exp = (int)(f32_bits(sc[(int64_t)(b * 2) * p.kv_heads + h]) >> 23);
            const int v_exp = (int)(f32_bits(sc[(int64_t)(b * 2 + 1) * p.kv_heads + h]) >> 23);
            f32x16 x[2];
            #pragma unroll
            for (int t = 0; t < 2; ++t) {
                #pragma unroll
                for (int r = 0; r < 16; ++r) x[t][r] = 0.0f;
                #pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const u32x4 a0 = *reinterpret_cast<const u32x4*>(&k_s[buf][(kaddr ^ (64 * j)) + t * 32 * D]);
                    const u32x4 a1 = *reinterpret_cast<const u32x4*>(&k_s[buf][(kaddr ^ (64 * j + 32)) + t * 32 * D]);
                    const i32x8 a = {(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
                    x[t] = mma(a, qh[j], x[t], k_exp, 127);
                    x[t] = mma(a, ql[j], x[t], k_exp, 123);
                }
            }
            const bool partial = r0 + kKvbBlock - 1 > wpos0;  // some row does not see every key
            if (partial) {
                #pragma unroll
                for (int t = 0; t < 2; ++t)
                    #pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (r0 + 32 * t + 8 * (r / 4) + 4 * half + r % 4 > pos) x[t][r] = f > 0.0f ? kNegInf : -kNegInf;
            }
            // f may be negative: the highest score is then that of the lowest product
            float top = kNegInf;
            #pragma unroll
            for (int t = 0; t < 2; ++t)
                #pragma unroll
                for (int r = 0; r < 16; ++r) {
                    x[t][r] *= f;
                    top = __builtin_fmaxf(top, x[t][r]);
                }
            const float c = __builtin_ceilf(pair_max(top)), base = c == kNegInf ? 0.0f : c - 8.0f;
            const float mn = __builtin_fmaxf(m, c);
            const float fade = __builtin_amdgcn_exp2f(mn == kNegInf ? 0.0f : m - mn);
            const float shift = __builtin_fmaxf(c - mn, -127.0f);  // c = mn = -inf: -127, with weights of zero
            m = mn;
            float sum = 0.0f;
            i32x8 ph, pl;
            #pragma unroll
            for (int t = 0; t < 2; ++t)
                #pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    float y[4];
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        y[i] = __builtin_amdgcn_exp2f(x[t][r + i] - base);
                        sum += y[i];
                    }
                    int a, d;
                    split4(y, a, d);
                    ph[4 * t + r / 4] = a;
                    pl[4 * t + r / 4] = d;
                }
            l = l * fade + sum * __builtin_amdgcn_exp2f(shift);
            if (__any(fade != 1.0f)) {
                #pragma unroll
                for (int i = 0; i < NT; ++i) acc[i] *= fade;
            }
            const int se = 127 + (int)shift, sl = se < 4 ? 0 : se - 4;
            #pragma unroll
            for (int i = 0; i < NT; ++i) {
                i32x8 a;
                #pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                        (__attribute__((address_space(3))) i32x2*)&v_s[buf][(vaddr ^ (32 * i)) + 16 * k * D]);
                    a[2 * k] = v[0];
                    a[2 * k + 1] = v[1];
                }
                acc[i] = mma(a, ph, acc[i], v_exp, se);
                acc[i] = mma(a, pl, acc[i], v_exp, sl);
            }
            if (partial && nan_s[buf] == b) {
                for (int t = 0; t < kKvbBlock; ++t) {
                    if (r0 + t >= s.n) break;
                    #pragma unroll
                    for (int i = 0; i < NT; ++i)
                        #pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const uint8_t code = vb[(r0 + t) * rowb + h * D + 32 * i + 8 * (r / 4) + 4 * half + r % 4];
                            if ((code & 0x7F) == 0x7F && r0 + t <= pos) acc[i][r] = __builtin_nanf("");
                        }
                }
            }
        }
        if (b + 1 < end) stage(b + 1, buf ^ 1);
    }

    l += __shfl_xor(l, 32);
    if (wrow0 + (lane & 31) > last) return;
    if (s.nsplit > 1) {
        const uint32_t slot = s.first_slot + (uint32_t)((tile * p.kv_heads + h) * s.nsplit + split);
        const int64_t at = (int64_t)slot * 128 + wave * 32 + (lane & 31);
        #pragma unroll
        for (int i = 0; i < NT; ++i)
            #pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4*>(p.part_o + at * D + 32 * i + 8 * (r / 4) + 4 * half) =
                    (f32x4){acc[i][r], acc[i][r + 1], acc[i][r + 2], acc[i][r + 3]};
        if (half == 0) *reinterpret_cast<f32x2*>(p.part_ml + at * 2) = (f32x2){m - 8.0f, l};
        return;
    }
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    const int64_t out = (s.t0 + token) * p.heads + (int64_t)h * G + row % G;
    #pragma unroll
    for (int i = 0; i < NT; ++i)
        #pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const bf16x2 a = __builtin_convertvector((f32x2){acc[i][r] * inv, acc[i][r + 1] * inv}, bf16x2);
            const bf16x2 b = __builtin_convertvector((f32x2){acc[i][r + 2] * inv, acc[i][r + 3] * inv}, bf16x2);
            *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.o) + out * D + 32 * i + 8 * (r / 4) + 4 * half) =
                (u32x2){__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
        }
    if (half == 0 && p.lse) p.lse[out] = (m - 8.0f + __builtin_amdgcn_logf(l)) * kLn2;
}

}  // namespace

hipError_t launch_kvb_prefill(const KvbAttendParams& p, hipStream_t stream) {
    const void* fn = p.d == 64    ? reinterpret_cast<const void*>(&prefill_kernel<64>)
                     : p.d == 128 ? reinterpret_cast<const void*>(&prefill_kernel<128>)
                                  : reinterpret_cast<const void*>(&prefill_kernel<256>);
    return launch_kernel(fn, dim3(p.wgs), dim3(kThreads), p, stream);
}

}  // namespace cap
