// Causal attention of many query rows over a block-scaled FP8 KV cache on gfx950
// (the formulas and the sharing of K and V by a group's heads: kvb_attend.hip).
//
// A workgroup takes 128 query rows of a KV head and walks the blocks; K and V of a block go
// through LDS, one barrier a block.  A wave has 32 of the rows; of 256 channels, where a
// row's outputs leave registers for one wave on a SIMD, two waves share the 32: each forms
// the scores and weights of half of the block's 64 keys, leaves the weights in LDS for the
// other, and multiplies all 64 with half of the channels of V, so that every SIMD has two.
// (161 tokens behind 16384, 32 heads on 4 of 256 channels, uncut: 575 us alone, 459 shared;
// of 128 channels, where two workgroups fit a CU, a prefill of 8192 takes 372 alone, 448 shared.)
//  * S^T = K Q^T on 32x32x16 bf16 tiles: the codes times their power-of-two scale are
//    exact in bf16, converted once for all waves on their way into LDS.  (FP8
//    instructions with Q split in two take the same matrix time, but their sums lose
//    what is small against the largest product: scores off by 1.6e-3 where a head's
//    channels differ in size.)
//  * O^T = V^T P^T on 32x32x64 FP8 tiles straight from the codes, with the scales as the
//    instruction's scale operands.  The weights of 32 rows are taken against their
//    own highest score, rounded up to an integer c in log2 units, w = 2^(x - c + 8) up to
//    2^8 (2^8.25 where scores near 2^23 are rounded), and split into two E4M3 rows,
//    w = hi + lo / 16 (relative 2^-8 at most, that of bf16, or 2^-21 of the 32's largest
//    weight where that is more); the instruction's sums lose 2^-12 of the sum of the
//    products' magnitudes at most.
//    2^(c - m) is the instruction's scale of a row, an exact power of two; m is the c of
//    the row's first block, raised only where a later one is 2^64 above: O and l are
//    floating, so their reference need not be the running maximum.  Beside values of V above 2^24
//    it is raised earlier, or above c, so that O stays below 2^127 for any rows of V.
//    Against bf16 operands that is the same matrix time (FP8 runs at twice the rate),
//    half the LDS traffic and no conversion of V.
//
// Half of a block's softmax stands between the matrix instructions of K Q^T of the block
// after it, the other half (the maximum first) between those of V^T P^T of the block before
// it, in slices that the scheduler must not move: a wave's vector instructions run beside
// its matrix instructions only where they are issued between them.
//
// 16384 tokens, 32 heads on 4 KV heads of 256 channels: 4.1 to 4.4 ms, 1000 to 1070 TFLOP/s
// (the library's bf16 product of 8192 reaches 1243).  Of the 4550 cycles of a block's step
// (counters) the matrix pipe is busy 2050; the rest are vector instructions beyond what stands beside
// them, reads of LDS and the barrier, at clocks that fall under matrix load.  A workgroup
// begins and ends in 5 us, which short prefills feel (512 tokens, 16 heads on 4 of 256: 25 us).
//
// A lane has one query row in both products and S^T's accumulators are P^T's
// operand: byte 4 j + i of lane half h is key 8 j + 4 h + i.  V's operand has its
// keys in the same order, read with the transposing 8-byte LDS read.  Rows in LDS
// are permuted in 16-byte units so that both reads are free of bank conflicts.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "kvb_device.h"

namespace cap {
namespace {

using dev::bf16x8;
using dev::rsrc_t;
using dev::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_inff();
constexpr float kLn2 = 0.6931471805599453f;

__device__ inline float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ inline uint32_t f32_bits(float f) { return __builtin_bit_cast(uint32_t, f); }
// The higher of the two lanes that share lane % 32.
__device__ inline float pair_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(f32_bits(x), f32_bits(x), false, false);
    return __builtin_fmaxf(bits_f32(r[0]), bits_f32(r[1]));
}
// The highest of a wave's lanes, in lane 63.
template <int CTRL, int ROWS>
__device__ inline uint32_t dpp_max(uint32_t x) {
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
    return x > y ? x : y;
}
__device__ inline uint32_t wave_max(uint32_t x) {
    x = dpp_max<0x118, 0xf>(dpp_max<0x114, 0xf>(dpp_max<0x112, 0xf>(dpp_max<0x111, 0xf>(x))));  // row_shr 1, 2, 4, 8
    return dpp_max<0x143, 0xc>(dpp_max<0x142, 0xa>(x));  // row_bcast 15 and 31
}
// Four values to four E4M3 codes, and their remainders times 16 to four more.
__device__ inline void split4(const float* y, int& hi, int& lo) {
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    i16x2 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, y[0] - a[0], y[1] - a[1], 0.0625f, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, y[2] - b[0], y[3] - b[1], 0.0625f, true);
    lo = __builtin_bit_cast(int, r);
}

__device__ inline f32x16 mma8(const i32x8& a, const i32x8& b, const f32x16& c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}
__device__ inline f32x16 mma16(const bf16x8& a, const bf16x8& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Eight codes times a power of two as bf16, exact.
__device__ inline u32x4 decode8(uint32_t w0, uint32_t w1, float scale) {
    return (u32x4){__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true))};
}

// Where the 16-byte unit `u` of row `key` lies in its row: u ^ the value.  LDS serves 256
// bytes at a time: of K one unit of 16 neighbouring rows (bf16, 2 D bytes), of V two
// neighbouring units of rows i and 8 + i, i = 0..3 or 4..7 (D bytes).
template <int D>
__device__ inline int swizzle_k(int key) { return D == 64 ? key >> 1 & 7 : key & 15; }
template <int D>
__device__ inline int swizzle_v(int key) {
    const int i = D == 256 ? (key & 3) | (key >> 3 & 1) << 2 : D == 128 ? (key >> 1 & 1) | (key >> 3 & 1) << 1 : key >> 3 & 1;
    return 2 * i;
}

// Exponent of V's scale and the rise of a block above the reference together (below).
constexpr int kRiseEnd = 206;

// Waves that share 32 query rows, and threads of a workgroup.
template <int D>
constexpr int kShare = D == 256 ? 2 : 1;
template <int D>
constexpr int kThreads = 256 * kShare<D>;

template <int D>
__global__ __launch_bounds__(kThreads<D>, 2) void prefill_kernel(const KvbAttendParams p) {
    constexpr int W = kShare<D>, S = 2 / W, NT = D / 32 / W;  // a wave's score tiles of 32 keys, its tiles of 32 channels of V
    constexpr int NJ = D / 32;
    constexpr int kUnits = D / 16, kRows = kThreads<D> / kUnits, kLoads = kKvbBlock / kRows;
    __shared__ __attribute__((aligned(1024))) uint8_t k_s[2][kKvbBlock * D * 2];  // bf16
    __shared__ __attribute__((aligned(1024))) uint8_t v_s[3][kKvbBlock * D];
    // of two waves that share their rows:
    __shared__ u32x4 p_s[2][4][2][2][64];  // weights: parity of the block, rows, half of the keys, hi or lo
    __shared__ float c_s[2][4][2][32];     // their references
    __shared__ int nan_s[3];
    __shared__ uint32_t top_s[kThreads<D> / 64];  // largest magnitude of q, of a wave's threads

    const KvbAttendSeq& s = p.seq[KVB_SEQ_OF(p, first_wg, blockIdx.x)];
    const uint32_t w = blockIdx.x - s.first_wg;
    const int G = p.heads / p.kv_heads;
    const uint32_t item = w / (uint32_t)s.nsplit;
    const int split = (int)(w - item * (uint32_t)s.nsplit);
    const int h = (int)(item % (uint32_t)p.kv_heads);
    const int64_t total = (int64_t)s.T * G, tiles = (total + 127) / 128;
    const int64_t tile = tiles - 1 - item / (uint32_t)p.kv_heads;  // the longest first
    const int tid = (int)threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), group = wave / W, part = wave % W;
    const int nblk = tile_blocks(s, tile * 128, 128, total, G), runs = tile_runs(s, nblk);
    if (split >= runs) return;
    const int64_t row0 = tile * 128, wrow0 = row0 + group * 32, last = total - 1;
    const int64_t row = wrow0 + (lane & 31) < last ? wrow0 + (lane & 31) : last;  // rows past the last repeat it
    const int64_t before = s.n - s.T, token = row_div(row, G), pos = before + token;     // the last key that the row sees
    // the wave's first position, the tile's
    const int64_t wpos0 = before + row_div(wrow0 < last ? wrow0 : last, G);
    const int64_t tpos0 = before + row_div(row0, G);

    const int rowb = p.kv_heads * D;
    const uint8_t* kb = reinterpret_cast<const uint8_t*>(s.k);
    const uint8_t* vb = reinterpret_cast<const uint8_t*>(s.v);
    const global_ptr<uint32_t> sc = (global_ptr<uint32_t>)s.scales;
    const int begin = split * s.per;
    const int end = begin + s.per < nblk ? begin + s.per : nblk;

    // Staging: thread tid moves unit tid % kUnits of rows tid / kUnits + i kRows.
    const int srow = tid / kUnits, sunit = tid % kUnits;
    const int svoff = srow * rowb + h * D + 16 * sunit;
    u32x4 ks[kLoads], vs[kLoads];
    auto fetch = [&](const uint8_t* base, int b, u32x4 (&x)[kLoads]) {
        const rsrc_t r = dev::make_rsrc_u32(base + (int64_t)b * kKvbBlock * rowb, (uint32_t)kKvbBlock * rowb);
        #pragma unroll
        for (int i = 0; i < kLoads; ++i) x[i] = __builtin_amdgcn_raw_buffer_load_b128(r, svoff, i * kRows * rowb, 0);
    };
    auto stage_k = [&](int buf, int i, float scale) {  // load i
        const int key = srow + i * kRows;
        uint8_t* dst = &k_s[buf][key * 2 * D];
        *reinterpret_cast<u32x4*>(dst + 16 * ((2 * sunit) ^ swizzle_k<D>(key))) = decode8(ks[i][0], ks[i][1], scale);
        *reinterpret_cast<u32x4*>(dst + 16 * ((2 * sunit + 1) ^ swizzle_k<D>(key))) = decode8(ks[i][2], ks[i][3], scale);
    };
    auto stage_v = [&](int b, int buf) {
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
            *reinterpret_cast<u32x4*>(&v_s[buf][key * D + 16 * (sunit ^ swizzle_v<D>(key))]) = vs[i];
        }
    };
    // The scales of 64 blocks from e0 on: lane i has those of block e0 + i.
    int e0 = begin;
    uint32_t k_scales = 0, v_scales = 0;
    auto load_scales = [&]() {
        const int64_t at = (int64_t)((e0 + lane < end ? e0 + lane : end - 1) * 2) * p.kv_heads + h;
        k_scales = sc[at];
        v_scales = sc[at + p.kv_heads];
    };
    auto k_scale = [&](int b) { return bits_f32((uint32_t)__builtin_amdgcn_readlane((int)k_scales, b - e0)); };
    auto v_exponent = [&](int b) { return __builtin_amdgcn_readlane((int)v_scales, b - e0) >> 23; };  // as the instruction takes it

    // addresses of a lane's reads; units and rows come in by xor and offset
    const int kaddr = (lane & 31) * 2 * D + 16 * (half ^ swizzle_k<D>(lane & 31));
    const int vkey = 4 * half + ((lane & 15) >> 1 & 3) + 8 * ((lane & 15) >> 3);
    const int vaddr = vkey * D + 16 * ((lane >> 4 & 1) ^ swizzle_v<D>(vkey)) + 8 * (lane & 1);
    // Rows of q and o are 2 D bytes, as those of K, and pass through its buffers, 16 bytes of a
    // row to a thread: straight from a lane's row an instruction takes a cycle a lane (the 16
    // loads of 8 waves 8600 cycles).
    constexpr int kRowUnits = D / 8, kRowPass = kThreads<D> / kRowUnits, kPasses = 128 / kRowPass;
    const int qrow = tid / kRowUnits, qunit = tid % kRowUnits;
    auto row_bytes = [&](int r) { return &k_s[0][0] + r * 2 * D + 16 * (qunit ^ swizzle_k<D>(r)); };
    auto token_of = [&](int64_t r) { return s.t0 + row_div(r, G); };
    auto head_of = [&](int64_t r) { return h * G + (int)row_mod(r, G); };

    // channels 16 s + 8 half .. + 7 of the lane's row; scores in log2 units are the products times f > 0
    bf16x8 q[D / 16];
    const float f = p.scale_log2 == 0.0f ? 1.0f : __builtin_fabsf(p.scale_log2);
    {
        u32x4 x[kPasses];
        #pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int64_t at = row0 + qrow + i * kRowPass, r = at < last ? at : last;
            x[i] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p.q) + token_of(r) * p.q_stride + (int64_t)head_of(r) * D * 2 + 16 * qunit);
        }
        fetch(kb, begin, ks);
        fetch(vb, begin, vs);
        load_scales();
        u16x2 top2 = {0, 0};
        #pragma unroll
        for (int i = 0; i < kPasses; ++i)
            #pragma unroll
            for (int k = 0; k < 4; ++k) top2 = __builtin_elementwise_max(top2, __builtin_bit_cast(u16x2, x[i][k] & 0x7FFF7FFFu));
        const uint32_t top = wave_max(top2[0] > top2[1] ? top2[0] : top2[1]);
        if (lane == 63) top_s[wave] = top;
        if (p.scale_log2 <= 0.0f) {  // a negative scale turns the rows' signs, zero makes them zero (but not their NaN)
            const float by = p.scale_log2 < 0.0f ? -1.0f : 0.0f;
            #pragma unroll
            for (int i = 0; i < kPasses; ++i)
                #pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float a = bits_f32(x[i][k] << 16), b = bits_f32(x[i][k] & 0xFFFF0000u);
                    x[i][k] = f32_bits(a * by) >> 16 | (f32_bits(b * by) & 0xFFFF0000u);
                }
        }
        #pragma unroll
        for (int i = 0; i < kPasses; ++i) *reinterpret_cast<u32x4*>(row_bytes(qrow + i * kRowPass)) = x[i];
    }
    if (tid < 3) nan_s[tid] = -1;
    dev::lds_barrier();
    #pragma unroll
    for (int i = 0; i < D / 16; ++i) q[i] = *reinterpret_cast<const bf16x8*>(&k_s[0][0] + (kaddr ^ (32 * i)) + group * 64 * D);
    // Whether a score of the blocks so far may reach 2^23 in log2 units: D products below 2^(exponent of q + 1),
    // 2^9 2^(exponent of the scale) and 2^(exponent of f + 1); exponents as they are stored, 127 too high.
    int far_from = 0;  // exponent of K's scale from which it may
    {
        uint32_t top = 0;
        #pragma unroll
        for (int i = 0; i < kThreads<D> / 64; ++i) top = top_s[i] > top ? top_s[i] : top;
        const int log2d = D == 64 ? 6 : D == 128 ? 7 : 8;
        far_from = __builtin_amdgcn_readfirstlane(23 + 3 * 127 - log2d - 1 - 9 - 1 - (int)(top >> 7) - (int)(f32_bits(f) >> 23));
    }
    int64_t whole = wpos0;  // keys up to here need nothing done to their scores; -1: all do
    auto check_scales = [&]() { whole = __any((int)(k_scales >> 23) >= far_from) ? -1 : whole; };

    auto read_k = [&](int buf, int t, int i) {  // keys 32 (part + t) .. + 31, channels 16 i .. + 15
        return *reinterpret_cast<const bf16x8*>(&k_s[buf][(kaddr ^ (32 * i)) + (part + t) * 64 * D]);
    };
    auto read_v = [&](int buf, int i) {  // channels 32 (part NT + i) .. + 31
        i32x8 a;
        #pragma unroll
        for (int k = 0; k < 4; ++k) {
            const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (__attribute__((address_space(3))) i32x2*)&v_s[buf][(vaddr ^ (32 * (part * NT + i))) + 16 * k * D]);
            a[2 * k] = v[0];
            a[2 * k + 1] = v[1];
        }
        return a;
    };

    f32x16 acc[NT], x[S], y[S];  // O^T; scores of block b and of block b + 1
    #pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] = (f32x16){};
    float m = kNegInf, l = 0.0f;
    float c = 0.0f, base = 0.0f, sum = 0.0f;  // of block b's softmax, whose first half is done when its step begins
    int ph[4 * S], pl[4 * S];                 // its weights, of the wave's keys

    float off = 0.0f;  // what block b's scores have been lowered by, in log2 units
    auto mask = [&](int b, f32x16 (&z)[S]) {
        const int64_t r0 = (int64_t)b * kKvbBlock;
        if (r0 + kKvbBlock - 1 <= whole) return;  // every row sees every key
        int sees = (int)(pos - r0 < kKvbBlock ? pos - r0 : kKvbBlock) - 4 * half - 32 * part;  // keys up to here
        asm volatile("" : "+v"(sees));  // rare: not to be computed ahead of the branch
        #pragma unroll
        for (int t = 0; t < S; ++t)
            #pragma unroll
            for (int r = 0; r < 16; ++r)
                if (32 * t + 8 * (r / 4) + r % 4 > sees) z[t][r] = kNegInf;
        if (whole >= 0) return;
        // x f - base is rounded once, c from the rounded product: from 2^24 on that differs by 1 and more, and a
        // weight above 2^8.8 has no code.  Scores as high as that are taken from their highest before the product.
        float high = z[0][0];
        #pragma unroll
        for (int t = 0; t < S; ++t)
            #pragma unroll
            for (int r = 0; r < 16; ++r) high = __builtin_fmaxf(high, z[t][r]);
        high = pair_max(high);
        off = __builtin_ceilf(high * f);
        if (__builtin_fabsf(off) < 0x1p23f || off == kNegInf) off = high = 0.0f;
        if (off == -kNegInf) high = __builtin_nanf("");  // beyond fp32
        #pragma unroll
        for (int t = 0; t < S; ++t)
            #pragma unroll
            for (int r = 0; r < 16; ++r) z[t][r] -= high;
    };
    auto weights = [&](int i) {  // of the wave's keys 8 i + 4 half .. + 3
        float e[4];
        #pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i / 4][4 * (i % 4) + k], f, -base));
        sum += (e[0] + e[1]) + (e[2] + e[3]);
        split4(e, ph[i], pl[i]);
    };
    auto highest = [&](int i) {  // of 8 of a lane's scores
        const int t = i / 2, r = 8 * (i % 2);
        const float u = __builtin_fmaxf(__builtin_fmaxf(x[t][r], x[t][r + 1]), x[t][r + 2]);
        const float v = __builtin_fmaxf(__builtin_fmaxf(x[t][r + 3], x[t][r + 4]), x[t][r + 5]);
        return __builtin_fmaxf(__builtin_fmaxf(u, v), __builtin_fmaxf(x[t][r + 6], x[t][r + 7]));
    };
    auto reference = [&](float top) {
        c = __builtin_ceilf(pair_max(top) * f);
        base = c == kNegInf ? 0.0f : c - 8.0f;
        c += off;
        sum = 0.0f;
    };
    // The first half of block b's softmax in slices 0..7, from its scores in y.
    float top = kNegInf;
    auto slice = [&](int u, int b) {
        if (u == 1) {
            #pragma unroll
            for (int t = 0; t < S; ++t) x[t] = y[t];
            mask(b, x);
            #pragma unroll
            for (int t = 0; t < S; ++t) asm volatile("" : "+v"(x[t]));
            top = S == 2 ? __builtin_fmaxf(highest(0), highest(1)) : highest(0);
        }
        if (u == 2) reference(__builtin_fmaxf(top, S == 2 ? __builtin_fmaxf(highest(2), highest(3)) : highest(1)));
        if (u >= 3 && u < 7 && (S == 2 || u % 2 == 0)) weights((u - 3) * S / 2);
    };

    // Block b's K lies in buffer (b - begin) & 1, its V in (b - begin) % 3.  The step
    // of block b reads K of b + 1, then V of b; in its first half K of b + 2 is
    // written, in its second V of b + 2, each where the block before the last was read.
    // Blocks past the end repeat the last one.
    auto clamp = [&](int b) { return b < end ? b : end - 1; };
    int ve = 127;  // exponent of V's scale of b
    check_scales();
    dev::lds_barrier();  // q has been read
    #pragma unroll
    for (int i = 0; i < kLoads; ++i) stage_k(0, i, k_scale(begin));
    stage_v(begin, 0);
    fetch(kb, clamp(begin + 1), ks);
    fetch(vb, clamp(begin + 1), vs);
    ve = v_exponent(begin);
    dev::lds_barrier();
    #pragma unroll
    for (int t = 0; t < S; ++t) {
        y[t] = (f32x16){};
        #pragma unroll
        for (int i = 0; i < D / 16; ++i) y[t] = mma16(read_k(0, t, i), q[i], y[t]);
    }
    #pragma unroll
    for (int i = 0; i < kLoads; ++i) stage_k(1, i, k_scale(clamp(begin + 1)));
    stage_v(clamp(begin + 1), 1);
    fetch(kb, clamp(begin + 2), ks);
    fetch(vb, clamp(begin + 2), vs);
    #pragma unroll
    for (int u = 0; u < 8; ++u) slice(u, begin);
    dev::lds_barrier();
    int vbuf = 0;
    for (int b = begin; b < end; ++b) {
        const int kbuf = (b - begin) & 1;
        const int next_ve = v_exponent(clamp(b + 1));
        if (b + 2 - e0 >= 64 && b + 2 < end) {
            e0 = b + 2;
            load_scales();
            check_scales();
        }
        const float next_scale = k_scale(clamp(b + 2));
        i32x8 v[S];
        {
            bf16x8 k[2 * S], next[2 * S];
            #pragma unroll
            for (int i = 0; i < 2 * S; ++i) k[i] = read_k(kbuf ^ 1, i % S, i / S);
            #pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (j + 1 < NJ) {
                    #pragma unroll
                    for (int i = 0; i < 2 * S; ++i) next[i] = read_k(kbuf ^ 1, i % S, 2 * (j + 1) + i / S);
                } else {
                    #pragma unroll
                    for (int i = 0; i < S; ++i) v[i] = read_v(vbuf, i);
                }
                #pragma unroll
                for (int i = 0; i < 2 * S; ++i) {
                    const int step = 2 * S * j + i, steps = 2 * S * NJ;
                    if (j == 0 && i < S) y[i] = (f32x16){};
                    y[i % S] = mma16(k[i], q[2 * j + i / S], y[i % S]);
                    #pragma unroll
                    for (int u = 0; u < 2 * S; ++u)
                        if (step == u * steps / (2 * S)) weights(2 * S + u);
                    #pragma unroll
                    for (int u = 0; u < kLoads; ++u)
                        if (step == (2 * u + 1) * steps / (2 * kLoads)) stage_k(kbuf, u, next_scale);
                    if (W == 2 && step == steps * 3 / 4) {
                        p_s[kbuf][group][part][0][lane] = (u32x4){(uint32_t)ph[0], (uint32_t)ph[1], (uint32_t)ph[2], (uint32_t)ph[3]};
                        p_s[kbuf][group][part][1][lane] = (u32x4){(uint32_t)pl[0], (uint32_t)pl[1], (uint32_t)pl[2], (uint32_t)pl[3]};
                        if (half == 0) c_s[kbuf][group][part][lane] = c;
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (j + 1 < NJ) {
                    #pragma unroll
                    for (int i = 0; i < 2 * S; ++i) k[i] = next[i];
                }
            }
        }
        // (what is needed late is not to be moved there)
        asm volatile("" : "+v"(sum));
        #pragma unroll
        for (int t = 0; t < S; ++t) asm volatile("" : "+v"(y[t]));
        i32x8 wh, wl;       // weights of the block's 64 rows
        float c0 = c, c1 = c;  // references of its two halves
        if constexpr (W == 1) {
            wh = (i32x8){ph[0], ph[1], ph[2], ph[3], ph[4], ph[5], ph[6], ph[7]};
            wl = (i32x8){pl[0], pl[1], pl[2], pl[3], pl[4], pl[5], pl[6], pl[7]};
            asm volatile("" : "+v"(wh), "+v"(wl));
        }
        dev::lds_barrier();
        fetch(kb, clamp(b + 3), ks);
        if constexpr (W == 2) {
            const u32x4 h0 = p_s[kbuf][group][0][0][lane], h1 = p_s[kbuf][group][1][0][lane];
            const u32x4 l0 = p_s[kbuf][group][0][1][lane], l1 = p_s[kbuf][group][1][1][lane];
            wh = (i32x8){(int)h0[0], (int)h0[1], (int)h0[2], (int)h0[3], (int)h1[0], (int)h1[1], (int)h1[2], (int)h1[3]};
            wl = (i32x8){(int)l0[0], (int)l0[1], (int)l0[2], (int)l0[3], (int)l1[0], (int)l1[1], (int)l1[2], (int)l1[3]};
            c0 = c_s[kbuf][group][0][lane & 31];
            c1 = c_s[kbuf][group][1][lane & 31];
        }
        const float cm = __builtin_fmaxf(c0, c1);
        // 2^31 products of weights up to 2^8 and values below 2^9 2^(ve - 127) stay below 2^127
        const float rise = (float)(kRiseEnd - ve < 64 ? kRiseEnd - ve : 64);
        if (m == kNegInf) m = cm;  // O and l are zero so far
        if (__any(cm - m > rise)) {
            float up = cm - m > rise ? cm + __builtin_fmaxf(-rise, 0.0f) : m;
            asm volatile("" : "+v"(up));  // rare: not to be computed ahead of the branch
            const float fade = up == m ? 1.0f : __builtin_amdgcn_exp2f(m - up);  // (a row that sees nothing yet: both -inf)
            #pragma unroll
            for (int i = 0; i < NT; ++i) acc[i] *= fade;
            l *= fade;
            m = up;
        }
        // The instruction's scales end at 2^-127, those of lo at 2^-123 of hi's: what is further below
        // weighs 2^-126 of the largest at most, but of large values that would show, and counts as none.
        if (__builtin_expect(ve > kRiseEnd - 64, 0)) {
            float d0 = c0 - m, d1 = c1 - m;
            asm volatile("" : "+v"(d0), "+v"(d1));  // (as above)
            #pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool none = (W == 2 && i >= 4 ? d1 : d0) < -123.0f;
                wh[i] = none ? 0 : wh[i];
                wl[i] = none ? 0 : wl[i];
            }
        }
        // no score: -127, with weights of zero
        l = __builtin_fmaf(sum, __builtin_amdgcn_exp2f(__builtin_fmaxf((part ? c1 : c0) - m, -127.0f)), l);
        // the instruction takes the scale of rows 0..31 from lanes 0..31, that of rows 32..63 from the others
        const int se = 127 + (int)__builtin_fmaxf((half ? c1 : c0) - m, -127.0f), sl = se < 4 ? 0 : se - 4;
        #pragma unroll
        for (int i = 0; i < NT; i += S) {
            i32x8 next[S];
            if (i + S < NT) {
                #pragma unroll
                for (int t = 0; t < S; ++t) next[t] = read_v(vbuf, i + S + t);
            }
            #pragma unroll
            for (int k = 0; k < 2 * S; ++k) {
                const int step = 2 * i + k, steps = 2 * NT;
                acc[i + k % S] = mma8(v[k % S], k < S ? wh : wl, acc[i + k % S], ve, k < S ? se : sl);
                #pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (u * steps / 8 == step) slice(u, b + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (i + S < NT) {
                #pragma unroll
                for (int t = 0; t < S; ++t) v[t] = next[t];
            }
        }
        asm volatile("" : "+v"(sum));
        {
            const int64_t r0 = (int64_t)b * kKvbBlock;
            if (r0 + kKvbBlock - 1 > tpos0 && nan_s[vbuf] == b) {
                for (int t = 0; t < kKvbBlock; ++t) {
                    if (r0 + t >= s.n) break;
                    #pragma unroll
                    for (int i = 0; i < NT; ++i)
                        #pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const uint8_t code = vb[(r0 + t) * rowb + h * D + 32 * (part * NT + i) + 8 * (r / 4) + 4 * half + r % 4];
                            if ((code & 0x7F) == 0x7F && r0 + t <= pos) acc[i][r] = __builtin_nanf("");
                        }
                }
            }
        }
        stage_v(clamp(b + 2), vbuf == 0 ? 2 : vbuf - 1);
        fetch(vb, clamp(b + 3), vs);
        ve = next_ve;
        vbuf = vbuf == 2 ? 0 : vbuf + 1;
    }

    l += __shfl_xor(l, 32);
    if constexpr (W == 2) {
        __syncthreads();  // the references have been read
        if (half == 0) c_s[0][group][part][lane] = l;
        __syncthreads();
        l = c_s[0][group][0][lane & 31] + c_s[0][group][1][lane & 31];
    }
    int orow = qrow, orow0 = lane & 31;
    asm volatile("" : "+v"(orow), "+v"(orow0));  // where rows lie: again, rather than held through the loop
    const int channel = 32 * NT * part + 4 * half;  // the lane's first
    if (runs > 1) {
        if (wrow0 + orow0 > last) return;
        const uint32_t slot = s.first_slot + (uint32_t)((tile * p.kv_heads + h) * s.nsplit + split);
        const int64_t at = (int64_t)slot * 128 + group * 32 + orow0;
        #pragma unroll
        for (int i = 0; i < NT; ++i)
            #pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4*>(p.part_o + at * D + channel + 32 * i + 8 * (r / 4)) =
                    (f32x4){acc[i][r], acc[i][r + 1], acc[i][r + 2], acc[i][r + 3]};
        if (lane < 32 && part == 0) *reinterpret_cast<f32x2*>(p.part_ml + at * 2) = (f32x2){m - 8.0f, l};
        return;
    }
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    const int out_addr = (kaddr ^ (16 * half)) + 8 * half + group * 64 * D;  // unit 0 of the lane's row, its half
    #pragma unroll
    for (int i = 0; i < NT; ++i)
        #pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const bf16x2 a = __builtin_convertvector((f32x2){acc[i][r] * inv, acc[i][r + 1] * inv}, bf16x2);
            const bf16x2 b = __builtin_convertvector((f32x2){acc[i][r + 2] * inv, acc[i][r + 3] * inv}, bf16x2);
            *reinterpret_cast<u32x2*>(&k_s[0][0] + (out_addr ^ (16 * (4 * (part * NT + i) + r / 4)))) =
                (u32x2){__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
        }
    if (lane < 32 && part == 0 && p.lse && wrow0 + orow0 <= last) {
        const int64_t r = wrow0 + orow0;
        p.lse[token_of(r) * p.heads + head_of(r)] = (m - 8.0f + __builtin_amdgcn_logf(l)) * kLn2;
    }
    dev::lds_barrier();
    #pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int64_t r = row0 + orow + i * kRowPass;
        if (r <= last)
            *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(p.o) + (token_of(r) * p.heads + head_of(r)) * D * 2 + 16 * qunit) =
                *reinterpret_cast<const u32x4*>(row_bytes(orow + i * kRowPass));
    }
}

}  // namespace

hipError_t launch_kvb_prefill(const KvbAttendParams& p, hipStream_t stream) {
    const void* fn = p.d == 64    ? reinterpret_cast<const void*>(&prefill_kernel<64>)
                     : p.d == 128 ? reinterpret_cast<const void*>(&prefill_kernel<128>)
                                  : reinterpret_cast<const void*>(&prefill_kernel<256>);
    return launch_kernel(fn, dim3(p.wgs), dim3(p.d == 256 ? kThreads<256> : kThreads<128>), p, stream);
}

}  // namespace cap
