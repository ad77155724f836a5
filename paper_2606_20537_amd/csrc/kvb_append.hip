// Append to a block-scaled FP8 KV cache on gfx950: bf16 rows of K and V to
// E4M3 codes, one power-of-two scale for each block of 64 rows and KV head.
//
// For a block's rows x (those held, the open block's old ones included):
//   e     = the smallest integer with max |x| <= 448 2^e (finite x only)
//   code  = E4M3(x 2^-e), nearest, ties to even
//   bounds: the lowest and the highest code of each channel (K only)
// A power of two loses nothing against max / 448: E4M3 keeps the same relative
// step over its range.  In return the products x 2^-e are exact, so every code
// is the correctly rounded one, and code 2^e is exact in bf16.
//
// A workgroup takes one block of one KV head, of K or of V: 64 x d values, held
// in registers between the maximum and the encoding, so that the rows are read
// once.  The open block is encoded again from its bf16 rows at every append:
// its codes, scale and bounds are a function of its rows alone, whatever calls
// brought them, also after a session went back to an earlier row.
#include <hip/hip_runtime.h>

#include "kvb_device.h"

namespace cap {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

__device__ inline float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ inline float elem(const u32x4& x, int i) {
    return bits_f32(i & 1 ? x[i / 2] & 0xFFFF0000u : x[i / 2] << 16);
}

// +-448 for anything larger, infinities included; NaN stays.
__device__ inline float saturate(float x) {
    return __builtin_fabsf(x) > 448.0f ? __builtin_copysignf(448.0f, x) : x;
}

// The scale's exponent: max = m 2^x with m in [0.5, 1), 448 = 0.875 2^9.
__device__ inline int scale_exponent(float amax) {
    const int x = __builtin_amdgcn_frexp_expf(amax);
    const float m = __builtin_amdgcn_frexp_mantf(amax);
    const int e = m <= 0.875f ? x - 9 : x - 8;
    return amax > 0.0f ? (e < -100 ? -100 : e > 119 ? 119 : e) : -100;
}

constexpr int kThreads = 256;

template <int D>
__global__ __launch_bounds__(kThreads) void append_kernel(const KvbAppendParams p) {
    constexpr int kPerRow = D / 8;               // threads of a row, 8 channels each
    constexpr int kRows = kThreads / kPerRow;    // rows of a pass
    constexpr int kPass = kKvbBlock / kRows;
    __shared__ float red[kThreads / 64];
    __shared__ float lo_s[kRows][D + 4], hi_s[kRows][D + 4];

    const KvbAppendSeq& s = p.seq[KVB_SEQ_OF(p, first_wg, blockIdx.x)];
    const uint32_t w = blockIdx.x - s.first_wg;
    const int side = (int)(w & 1), h = (int)((w >> 1) % (uint32_t)p.kv_heads);
    const int64_t held = s.n - s.T;              // rows before the append
    const int64_t b0 = held / kKvbBlock, b = b0 + (w >> 1) / (uint32_t)p.kv_heads;
    const int64_t r0 = b * kKvbBlock;
    const int rows = (int)(s.n - r0 < kKvbBlock ? s.n - r0 : kKvbBlock);
    const int old = (int)(held > r0 ? held - r0 : 0);  // rows of the block that are in `open`
    const int tid = (int)threadIdx.x, col = tid % kPerRow * 8, row = tid / kPerRow;
    const int64_t rowb = (int64_t)p.kv_heads * D;      // codes of a row
    uint8_t* open = reinterpret_cast<uint8_t*>(s.open) + ((int64_t)side * kKvbBlock * rowb + (int64_t)h * D + col) * 2;
    const uint8_t* fresh = static_cast<const uint8_t*>(side ? p.v_new : p.k_new) + ((int64_t)h * D + col) * 2;
    const int64_t stride = side ? p.v_stride : p.k_stride;
    const int64_t token0 = s.t0 + r0 - held;           // packed token of row r0

    u32x4 x[kPass];
    #pragma unroll
    for (int i = 0; i < kPass; ++i) {
        const int r = row + i * kRows;
        x[i] = (u32x4){0, 0, 0, 0};
        if (r < rows)
            x[i] = *reinterpret_cast<const u32x4*>(r < old ? open + r * rowb * 2 : fresh + (token0 + r) * stride);
    }
    float amax = 0.0f;
    bool special = false;  // infinities or NaN
    #pragma unroll
    for (int i = 0; i < kPass; ++i)
        #pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float a = __builtin_fabsf(elem(x[i], c));
            if (a < __builtin_inff()) amax = __builtin_fmaxf(amax, a); else special = true;
        }
    #pragma unroll
    for (int o = 32; o > 0; o >>= 1) amax = __builtin_fmaxf(amax, __shfl_xor(amax, o));
    if ((tid & 63) == 0) red[tid / 64] = amax;
    special = __syncthreads_or(special);  // also: every read of `open` is done
    amax = __builtin_fmaxf(__builtin_fmaxf(red[0], red[1]), __builtin_fmaxf(red[2], red[3]));
    const int e = scale_exponent(amax);
    const float mul = bits_f32((uint32_t)(127 - e) << 23);  // 2^-e
    uint8_t* codes = reinterpret_cast<uint8_t*>(side ? s.v : s.k) + r0 * rowb + (int64_t)h * D + col;
    float mn[8], mx[8];
    uint32_t nan = 0;
    #pragma unroll
    for (int c = 0; c < 8; ++c) { mn[c] = __builtin_inff(); mx[c] = -__builtin_inff(); }
    #pragma unroll
    for (int i = 0; i < kPass; ++i) {
        const int r = row + i * kRows;
        if (r < rows) {
            float y[8];
            #pragma unroll
            for (int c = 0; c < 8; ++c) {
                y[c] = elem(x[i], c) * mul;
                if (special || e == 119) {
                    y[c] = saturate(y[c]);
                    if (y[c] != y[c]) nan |= 1u << c;
                }
                mn[c] = __builtin_fminf(mn[c], y[c]);
                mx[c] = __builtin_fmaxf(mx[c], y[c]);
            }
            u32x2 out;
            #pragma unroll
            for (int k = 0; k < 2; ++k)
                out[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(
                    y[4 * k + 2], y[4 * k + 3], __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * k], y[4 * k + 1], 0, false), true);
            *reinterpret_cast<u32x2*>(codes + r * rowb) = out;
        }
    }
    if (tid == 0)
        reinterpret_cast<float*>(s.scales)[(b * 2 + side) * p.kv_heads + h] = bits_f32((uint32_t)(127 + e) << 23);
    if (side == 0 && s.bounds) {
        #pragma unroll
        for (int c = 0; c < 8; ++c) {
            lo_s[row][col + c] = nan >> c & 1 ? __builtin_nanf("") : mn[c];
            hi_s[row][col + c] = mx[c];
        }
        __syncthreads();
        if (tid < D / 2) {
            float a[2], z[2];
            #pragma unroll
            for (int c = 0; c < 2; ++c) {
                a[c] = __builtin_inff();
                z[c] = -__builtin_inff();
                bool bad = false;
                for (int r = 0; r < kRows; ++r) {
                    const float u = lo_s[r][2 * tid + c];
                    bad |= u != u;
                    a[c] = __builtin_fminf(a[c], u);
                    z[c] = __builtin_fmaxf(z[c], hi_s[r][2 * tid + c]);
                }
                // the sum makes one zero of the two; a NaN in a channel is both of its bounds
                a[c] = bad ? __builtin_nanf("") : a[c] + 0.0f;
                z[c] = bad ? __builtin_nanf("") : z[c] + 0.0f;
            }
            uint8_t* bounds = reinterpret_cast<uint8_t*>(s.bounds) + (b * 2 * p.kv_heads + h) * D + 2 * tid;
            *reinterpret_cast<uint16_t*>(bounds) = (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(a[0], a[1], 0, false);
            *reinterpret_cast<uint16_t*>(bounds + rowb) = (uint16_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
        }
    }
    // The rows of the block that is open after the append.  The workgroup that
    // read the old ones writes the new ones, behind the barrier above.
    const int left = (int)(s.n % kKvbBlock);
    if (b == b0 && left) {
        const int64_t last0 = s.n - left;
        for (int r = row; r < left; r += kRows)
            if (last0 + r >= held)
                *reinterpret_cast<u32x4*>(open + r * rowb * 2) =
                    *reinterpret_cast<const u32x4*>(fresh + (s.t0 + last0 + r - held) * stride);
    }
}

}  // namespace

hipError_t launch_kvb_append(const KvbAppendParams& p, hipStream_t stream) {
    if (p.wgs == 0) return hipSuccess;
    const void* fn = p.d == 64    ? reinterpret_cast<const void*>(&append_kernel<64>)
                     : p.d == 128 ? reinterpret_cast<const void*>(&append_kernel<128>)
                                  : reinterpret_cast<const void*>(&append_kernel<256>);
    return launch_kernel(fn, dim3(p.wgs), dim3(kThreads), p, stream);
}

}  // namespace cap
