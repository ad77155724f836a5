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
//
// Bound by memory: 16384 rows x 4 heads x 256 channels, 101 MB, 17.5 us (5.8 TB/s read and
// written; a copy of 1 GiB 5.2).  With the maximum, the bounds and the conversion in 32
// bits an element took some 12 instructions and the call 26 us; now maximum and bounds are
// 16-bit integers, two at a time, and the conversion one instruction for two values.
#include <hip/hip_runtime.h>

#include "kvb_device.h"

namespace cap {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ inline float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ inline float elem(const u32x4& x, int i) {
    return bits_f32(i & 1 ? x[i / 2] & 0xFFFF0000u : x[i / 2] << 16);
}

// +-448 for anything larger, infinities included; NaN stays.
__device__ inline float saturate(float x) {
    return __builtin_fabsf(x) > 448.0f ? __builtin_copysignf(448.0f, x) : x;
}

// (by value: __builtin_bit_cast of a vector's element reads the vector's first one)
__device__ inline bf16x2 pair(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }

// Two bf16 values in one word, as 16-bit integers in the order of the values (and back:
// the map is its own inverse).
__device__ inline i16x2 ordered(uint32_t w) {
    const i16x2 x = __builtin_bit_cast(i16x2, w);
    return x ^ ((x >> 15) & (i16x2){0x7FFF, 0x7FFF});
}
__device__ inline i16x2 min2(i16x2 a, i16x2 b) { return __builtin_elementwise_min(a, b); }
__device__ inline i16x2 max2(i16x2 a, i16x2 b) { return __builtin_elementwise_max(a, b); }

// The scale's exponent: max = m 2^x with m in [0.5, 1), 448 = 0.875 2^9.
__device__ inline int scale_exponent(float amax) {
    const int x = __builtin_amdgcn_frexp_expf(amax);
    const float m = __builtin_amdgcn_frexp_mantf(amax);
    const int e = m <= 0.875f ? x - 9 : x - 8;
    return amax > 0.0f ? (e < -100 ? -100 : e > 119 ? 119 : e) : -100;
}

// Two codes with +0 for -0 (what a small negative value rounds to).
__device__ inline uint16_t one_zero(uint32_t w) {
    if ((w & 0xFFu) == 0x80u) w &= 0xFF00u;
    if ((w & 0xFF00u) == 0x8000u) w &= 0xFFu;
    return (uint16_t)w;
}

constexpr int kThreads = 256;

template <int D, int N>
__global__ __launch_bounds__(kThreads, 4) void append_kernel(const KvbAppendTable<N> p) {
    constexpr int kPerRow = D / 8;               // threads of a row, 8 channels each
    constexpr int kRows = kThreads / kPerRow;    // rows of a pass
    constexpr int kPass = kKvbBlock / kRows;
    __shared__ uint32_t red[kThreads / 64];
    __shared__ i16x2 lo_s[kRows][D / 2 + 4], hi_s[kRows][D / 2 + 4];
    __shared__ uint8_t nan_s[D];

    const uint32_t block = kvb_block();
    if (block >= p.wgs) return;
    const KvbAppendSeq& s = p.seq[KVB_SEQ_OF(p, first_wg, block)];
    const uint32_t w = block - s.first_wg;
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

    auto at = [&](int r) { return reinterpret_cast<const u32x4*>(r < old ? open + r * rowb * 2 : fresh + (token0 + r) * stride); };
    u32x4 x[kPass];
    #pragma unroll
    for (int i = 0; i < kPass; ++i) {
        const int r = row + i * kRows;
        x[i] = (u32x4){0, 0, 0, 0};
        if (r < rows) x[i] = *at(r);
    }
    // The largest magnitude, as the integer that its bits are (rows that are not there: 0).
    u16x2 top2 = {0, 0};
    #pragma unroll
    for (int i = 0; i < kPass; ++i)
        #pragma unroll
        for (int k = 0; k < 4; ++k) top2 = __builtin_elementwise_max(top2, __builtin_bit_cast(u16x2, x[i][k] & 0x7FFF7FFFu));
    uint32_t top = top2[0] > top2[1] ? top2[0] : top2[1];
    #pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const uint32_t u = __shfl_xor(top, o);
        top = u > top ? u : top;
    }
    if ((tid & 63) == 0) red[tid / 64] = top;
    if (tid < D) nan_s[tid] = 0;
    __syncthreads();  // also: every read of `open` is done
    #pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) top = red[i] > top ? red[i] : top;
    const bool special = top >= 0x7F80;  // infinities or NaN
    if (special) {                       // the maximum without them
        uint32_t u = 0;
        #pragma unroll 1
        for (int r = row; r < rows; r += kRows) {
            const u32x4 y = *at(r);
            #pragma unroll
            for (int c = 0; c < 8; ++c) {
                const uint32_t a = (c & 1 ? y[c / 2] >> 16 : y[c / 2]) & 0x7FFF;
                if (a < 0x7F80 && a > u) u = a;
                if (a > 0x7F80) nan_s[col + c] = 1;
            }
        }
        #pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const uint32_t v = __shfl_xor(u, o);
            u = v > u ? v : u;
        }
        __syncthreads();
        if ((tid & 63) == 0) red[tid / 64] = u;
        __syncthreads();
        top = 0;
        #pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) top = red[i] > top ? red[i] : top;
    }
    const int e = scale_exponent(bits_f32(top << 16));
    const float scale = bits_f32((uint32_t)(127 + e) << 23), mul = bits_f32((uint32_t)(127 - e) << 23);
    const bool beyond = special || e == 119;  // values that saturate
    uint8_t* codes = reinterpret_cast<uint8_t*>(side ? s.v : s.k) + r0 * rowb + (int64_t)h * D + col;
    i16x2 mn[4], mx[4];
    #pragma unroll
    for (int k = 0; k < 4; ++k) {
        mn[k] = (i16x2){0x7FFF, 0x7FFF};
        mx[k] = (i16x2){-0x8000, -0x8000};
    }
    auto bound = [&](const u32x4& y) {
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            const i16x2 o = ordered(y[k]);
            mn[k] = min2(mn[k], o);
            mx[k] = max2(mx[k], o);
        }
    };
    if (!beyond) {
        #pragma unroll
        for (int i = 0; i < kPass; ++i) {
            const int r = row + i * kRows;
            if (r >= rows) continue;
            u32x2 out;
            #pragma unroll
            for (int k = 0; k < 2; ++k) {
                i16x2 w = {0, 0};
                w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, pair(x[i][2 * k]), scale, false);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, pair(x[i][2 * k + 1]), scale, true);
                out[k] = __builtin_bit_cast(uint32_t, w);
            }
            *reinterpret_cast<u32x2*>(codes + r * rowb) = out;
            if (side == 0) bound(x[i]);
        }
    } else {  // rare: read again
        #pragma unroll 1
        for (int r = row; r < rows; r += kRows) {
            const u32x4 y = *at(r);
            u32x2 out;
            #pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int z = __builtin_amdgcn_cvt_pk_fp8_f32(saturate(elem(y, 4 * k) * mul), saturate(elem(y, 4 * k + 1) * mul), 0, false);
                out[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(saturate(elem(y, 4 * k + 2) * mul), saturate(elem(y, 4 * k + 3) * mul), z, true);
            }
            *reinterpret_cast<u32x2*>(codes + r * rowb) = out;
            if (side == 0) bound(y);
        }
    }
    if (tid == 0) reinterpret_cast<float*>(s.scales)[(b * 2 + side) * p.kv_heads + h] = scale;
    if (side == 0 && s.bounds) {
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            lo_s[row][col / 2 + k] = mn[k];
            hi_s[row][col / 2 + k] = mx[k];
        }
        __syncthreads();
        if (tid < D / 2) {
            i16x2 a = lo_s[0][tid], z = hi_s[0][tid];
            #pragma unroll
            for (int r = 1; r < kRows; ++r) {
                a = min2(a, lo_s[r][tid]);
                z = max2(z, hi_s[r][tid]);
            }
            const uint32_t lo = __builtin_bit_cast(uint32_t, ordered(__builtin_bit_cast(uint32_t, a)));
            const uint32_t hi = __builtin_bit_cast(uint32_t, ordered(__builtin_bit_cast(uint32_t, z)));
            float y[4] = {bits_f32(lo << 16), bits_f32(lo & 0xFFFF0000u), bits_f32(hi << 16), bits_f32(hi & 0xFFFF0000u)};
            #pragma unroll
            for (int c = 0; c < 4; ++c)  // a NaN in a channel is both of its bounds
                y[c] = nan_s[2 * tid + (c & 1)] ? __builtin_nanf("") : saturate(y[c] * mul);
            uint8_t* bounds = reinterpret_cast<uint8_t*>(s.bounds) + (b * 2 * p.kv_heads + h) * D + 2 * tid;
            *reinterpret_cast<uint16_t*>(bounds) = one_zero((uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false));
            *reinterpret_cast<uint16_t*>(bounds + rowb) = one_zero((uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], 0, false));
        }
    }
    // The rows of the block that is open after the append.  The workgroup that
    // read the old ones writes the new ones, behind a barrier.
    if (beyond) __syncthreads();  // `open` has been read again
    const int left = (int)(s.n % kKvbBlock);
    if (b == b0 && left) {
        const int64_t last0 = s.n - left;
        for (int r = row; r < left; r += kRows)
            if (last0 + r >= held)
                *reinterpret_cast<u32x4*>(open + r * rowb * 2) =
                    *reinterpret_cast<const u32x4*>(fresh + (s.t0 + last0 + r - held) * stride);
    }
}

template <int D>
hipError_t launch(const KvbAppendParams& p, hipStream_t stream) {
    return launch_kvb<KvbAppendTable>(reinterpret_cast<const void*>(&append_kernel<D, kKvbFew>),
                                      reinterpret_cast<const void*>(&append_kernel<D, KVB_MAX_SEQ>), kvb_grid(p.wgs), dim3(kThreads), p, stream);
}

}  // namespace

hipError_t launch_kvb_append(const KvbAppendParams& p, hipStream_t stream) {
    if (p.wgs == 0) return hipSuccess;
    return p.d == 64 ? launch<64>(p, stream) : p.d == 128 ? launch<128>(p, stream) : launch<256>(p, stream);
}

}  // namespace cap
