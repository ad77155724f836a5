// Causal attention over a block-scaled FP8 KV cache on gfx950.
//
//   x_j = scale q . k_j,  o = sum_j exp(x_j - m) v_j / l,  m = max x_j,
//   l = sum_j exp(x_j - m),  lse = m + log l,  over the rows j that the query
//   sees (j <= its position; with a block list, of the listed blocks)
//
// in one pass over K and V with a running m and l.  The query rows of a KV head
// (tokens x query heads of the group) share its K and V: 16 of them are the
// columns of the matrix instructions, keys and channels the rows.
//  * S^T = K Q^T on 16x16x128 FP8 tiles straight from the codes.  A bf16 query
//    row is split into two E4M3 rows, q 2^-e = hi + lo / 16 (e: the row's largest
//    value falls in [128, 256)): 4 + 4 bits are bf16's 8, what is lost is below
//    2^-22 of the row's largest value.
//  * O^T = V^T P^T on 16x16x32 bf16 tiles: codes times the block's power-of-two
//    scale are exact in bf16, P is rounded to bf16 (relative 2^-8 at most, as
//    the output is); l sums the unrounded P in 32 bits.
// Both products leave a lane with one query row (lane % 16), so maximum, sum and
// correction need no value of another row, and S^T's accumulators are P^T's
// operand: lane group g holds keys 4g..4g+3 and 16+4g..16+4g+3 of 32, and loads
// V's rows in that order.  A lane reads d / 16 contiguous bytes of eight rows and
// transposes them in registers.  K and V go from memory to registers; LDS only
// joins the four waves, which take 32 rows of the cache in turn.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "kvb.h"

namespace cap {
namespace {

using dev::bf16x8;
using dev::f32x4;
using dev::rsrc_t;
using dev::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr float kNegInf = -__builtin_inff();
constexpr float kLn2 = 0.6931471805599453f;

__device__ inline float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ inline uint32_t f32_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

// Maximum / sum over the four lanes that share lane % 16.
__device__ inline float group_max(float x) {
    x = __builtin_fmaxf(x, __shfl_xor(x, 16));
    return __builtin_fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float group_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// 0x80 in exactly the bytes of w that hold a NaN code (0x7F or 0xFF).
__device__ inline uint32_t nan_bytes(uint32_t w) {
    return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// 4x4 bytes: out[c] = byte c of in[0..3].
__device__ inline void transpose4(const uint32_t* in, uint32_t* out) {
    const uint32_t a = __builtin_amdgcn_perm(in[1], in[0], 0x05010400u);  // 0.0 1.0 0.1 1.1
    const uint32_t b = __builtin_amdgcn_perm(in[1], in[0], 0x07030602u);  // 0.2 1.2 0.3 1.3
    const uint32_t c = __builtin_amdgcn_perm(in[3], in[2], 0x05010400u);
    const uint32_t d = __builtin_amdgcn_perm(in[3], in[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Four codes times a power of two as bf16, exact.
__device__ inline void decode4(uint32_t w, float scale, bf16x8& v, int at) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
    v[at] = a[0];
    v[at + 1] = a[1];
    v[at + 2] = b[0];
    v[at + 3] = b[1];
}

// A query row's two E4M3 rows in operand order, and the power of two that
// belongs to them.  A lane holds channels 64 j + 16 g .. + 15 of its row.
template <int D>
struct Query {
    static constexpr int kSteps = D == 64 ? 1 : D / 128;
    i32x8 hi[kSteps], lo[D == 64 ? 1 : kSteps];  // D == 64: hi and lo in one operand
    float scale;

    __device__ void load(const uint8_t* row, int g) {
        u32x4 x[D / 32];
        float amax = 0.0f;
        #pragma unroll
        for (int j = 0; j < D / 64; ++j)
            #pragma unroll
            for (int c = 0; c < 2; ++c)
                x[2 * j + c] = *reinterpret_cast<const u32x4*>(row + (64 * j + 16 * g + 8 * c) * 2);
        #pragma unroll
        for (int i = 0; i < D / 32; ++i)
            #pragma unroll
            for (int k = 0; k < 4; ++k)
                amax = __builtin_fmaxf(amax, __builtin_fmaxf(__builtin_fabsf(bits_f32(x[i][k] << 16)),
                                                             __builtin_fabsf(bits_f32(x[i][k] & 0xFFFF0000u))));
        amax = group_max(amax);
        int e = (int)(f32_bits(amax) >> 23) - 127 - 7;  // amax 2^-e in [128, 256)
        e = e < -100 ? -100 : e;
        const float mul = bits_f32((uint32_t)(127 - e) << 23);  // an infinity stays one, and becomes NaN below
        scale = bits_f32((uint32_t)(127 + e) << 23);
        #pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            #pragma unroll
            for (int w = 0; w < 4; ++w) {
                float y[4], z[4];
                #pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t u = x[2 * j + w / 2][2 * (w % 2) + k];
                    y[2 * k] = bits_f32(u << 16) * mul;
                    y[2 * k + 1] = bits_f32(u & 0xFFFF0000u) * mul;
                }
                const int a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
                const f32x2 b0 = __builtin_amdgcn_cvt_pk_f32_fp8(a, false), b1 = __builtin_amdgcn_cvt_pk_f32_fp8(a, true);
                z[0] = (y[0] - b0[0]) * 16.0f;
                z[1] = (y[1] - b0[1]) * 16.0f;
                z[2] = (y[2] - b1[0]) * 16.0f;
                z[3] = (y[3] - b1[1]) * 16.0f;
                const int r = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false), true);
                if (D == 64) {
                    hi[0][w] = a;
                    hi[0][4 + w] = r;
                } else {
                    hi[j / 2][4 * (j % 2) + w] = a;
                    lo[j / 2][4 * (j % 2) + w] = r;
                }
            }
        }
    }
};

// 16 keys (lane % 16: a key, chunk j of 16 bytes: channels 64 j + 16 g ..) against 16 query rows.
template <int D>
__device__ inline f32x4 scores(const u32x4* k, const Query<D>& q, int lane) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (D == 64) {
        // channels 0..63 twice: against hi, and against lo with 2^-4 from lane groups 2 and 3, whose
        // scales belong to the operand's second half
        i32x8 a;
        #pragma unroll
        for (int w = 0; w < 4; ++w) a[w] = a[4 + w] = (int)k[0][w];
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.hi[0], s, 0, 0, 0, 127, 0, lane < 32 ? 127 : 123);
    }
    #pragma unroll
    for (int i = 0; i < Query<D>::kSteps; ++i) {
        i32x8 a;
        #pragma unroll
        for (int w = 0; w < 4; ++w) {
            a[w] = (int)k[2 * i][w];
            a[4 + w] = (int)k[2 * i + 1][w];
        }
        s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.hi[i], s, 0, 0, 0, 127, 0, 127);
        s = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.lo[i], s, 0, 0, 0, 127, 0, 123);
    }
    return s;
}

// A lane's bytes of one row of V.
template <int VB>
struct VBytes { uint32_t w[VB / 4]; };
template <int VB>
__device__ inline VBytes<VB> load_v(rsrc_t r, int voff, int soff) {
    VBytes<VB> x;
    if constexpr (VB == 16) {
        const u32x4 t = __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 0);
        #pragma unroll
        for (int i = 0; i < 4; ++i) x.w[i] = t[i];
    } else if constexpr (VB == 8) {
        const u32x2 t = __builtin_amdgcn_raw_buffer_load_b64(r, voff, soff, 0);
        x.w[0] = t[0];
        x.w[1] = t[1];
    } else {
        x.w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, voff, soff, 0);
    }
    return x;
}

template <int D, bool SPARSE>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(const KvbAttendParams p) {
    constexpr int VB = D / 16, NJ = D / 64;
    constexpr int kPitch = D + 4;
    __shared__ float o_s[4][16][kPitch];
    __shared__ float ml_s[4][16][2];

    int lo = 0, hi = p.n_seq - 1;  // last s with first_wg <= blockIdx.x
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.seq[mid].first_wg <= blockIdx.x) lo = mid; else hi = mid - 1;
    }
    const KvbAttendSeq& s = p.seq[__builtin_amdgcn_readfirstlane(lo)];
    const uint32_t w = blockIdx.x - s.first_wg;
    const int G = p.heads / p.kv_heads;
    const uint32_t item = w / (uint32_t)s.nsplit;  // (tile, kv head)
    const int split = (int)(w - item * (uint32_t)s.nsplit);
    const int h = (int)(item % (uint32_t)p.kv_heads);
    const int64_t tile = item / (uint32_t)p.kv_heads;
    // the tile's rows: `rows` of them from row r0 of the sequence, or of token `token` (sparse)
    int64_t r0, total;
    int64_t token = 0;
    if (SPARSE) {
        const int per = (G + 15) / 16;
        token = tile / per;
        r0 = (tile - token * per) * 16;
        total = G;
    } else {
        r0 = tile * 16;
        total = (int64_t)s.T * G;
    }
    const int rows = (int)(total - r0 < 16 ? total - r0 : 16);
    const int tid = (int)threadIdx.x, lane = tid & 63, li = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = r0 + (li < rows ? li : rows - 1);  // rows past the last repeat it
    const int64_t my_token = SPARSE ? token : row / G;
    const int64_t pos = s.n - s.T + my_token;              // the last key that the row sees
    const int64_t pos0 = s.n - s.T + (SPARSE ? token : r0 / G), pos1 = s.n - s.T + (SPARSE ? token : (r0 + rows - 1) / G);

    Query<D> q;
    q.load(static_cast<const uint8_t*>(p.q) + (s.t0 + my_token) * p.q_stride + ((int64_t)h * G + row % G) * D * 2, g);
    const float row_scale = q.scale * p.scale_log2;

    const int rowb = p.kv_heads * D;
    const uint8_t* kb = reinterpret_cast<const uint8_t*>(s.k);
    const uint8_t* vb = reinterpret_cast<const uint8_t*>(s.v);
    const float* sc = reinterpret_cast<const float*>(s.scales);
    const int kvoff = li * rowb + h * D + 16 * g, vvoff = 4 * g * rowb + h * D + li * VB;
    const int32_t* list = SPARSE ? p.idx + ((s.t0 + token) * p.kv_heads + h) * p.n_sel : nullptr;

    const int nblk = SPARSE ? p.n_sel : (int)(pos1 / kKvbBlock + 1);
    const int begin = split * s.per, end = begin + s.per < nblk ? begin + s.per : nblk;
    const int units = 2 * (end - begin);

    // first row of unit u (32 rows); -1: nothing there (an entry that names no visible block)
    auto unit_row = [&](int u) -> int64_t {
        if (u >= units) return -1;
        int64_t b = begin + (u >> 1);
        if (SPARSE) {
            b = __builtin_amdgcn_readfirstlane(list[b]);
            if (b < 0 || b * kKvbBlock > pos) return -1;
        }
        const int64_t r = b * kKvbBlock + 32 * (u & 1);
        return r <= pos1 ? r : -1;
    };
    auto load_k = [&](int64_t r, u32x4 (&k)[2][NJ]) {
        const rsrc_t rk = dev::make_rsrc_u32(kb + r * rowb, 32u * rowb);
        #pragma unroll
        for (int t = 0; t < 2; ++t)
            #pragma unroll
            for (int j = 0; j < NJ; ++j)
                k[t][j] = __builtin_amdgcn_raw_buffer_load_b128(rk, kvoff + 64 * j, t * 16 * rowb, 0);
    };

    f32x4 acc[VB];
    #pragma unroll
    for (int c = 0; c < VB; ++c) acc[c] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    float m = kNegInf, l = 0.0f;

    u32x4 k[2][NJ];
    int64_t r = unit_row(wave);
    if (r >= 0) load_k(r, k);
    for (int u = wave; u < units; u += 4) {
        const int64_t next = unit_row(u + 4);
        if (r >= 0) {
            VBytes<VB> v[8];
            const rsrc_t rv = dev::make_rsrc_u32(vb + r * rowb, 32u * rowb);
            #pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = load_v<VB>(rv, vvoff, (e < 4 ? e : 12 + e) * rowb);
            const int64_t b = r / kKvbBlock;
            const float k_scale = sc[(b * 2) * p.kv_heads + h], v_scale = sc[(b * 2 + 1) * p.kv_heads + h];
            const f32x4 s0 = scores<D>(k[0], q, lane), s1 = scores<D>(k[1], q, lane);
            if (next >= 0) load_k(next, k);
            float x[8];
            #pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = s0[e] * (row_scale * k_scale);
                x[4 + e] = s1[e] * (row_scale * k_scale);
            }
            const bool partial = r + 31 > pos0;  // some row does not see every key
            bool nan_seen = false;
            if (partial) {
                #pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t key = r + 4 * g + (e < 4 ? e : 12 + e);
                    if (key > pos) x[e] = kNegInf;
                    // NaN in V times a weight of zero would be NaN: such codes go, and are put back below
                    #pragma unroll
                    for (int i = 0; i < VB / 4; ++i) {
                        const uint32_t bad = nan_bytes(v[e].w[i]);
                        nan_seen |= bad != 0 && key < s.n;
                        v[e].w[i] &= ~(bad | (bad - (bad >> 7)));
                    }
                }
            }
            float top = __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(x[0], x[1]), __builtin_fmaxf(x[2], x[3])),
                                        __builtin_fmaxf(__builtin_fmaxf(x[4], x[5]), __builtin_fmaxf(x[6], x[7])));
            top = __builtin_fmaxf(m, group_max(top));
            const float base = top == kNegInf ? 0.0f : top;
            const float fade = __builtin_amdgcn_exp2f(m - base);
            m = top;
            float sum = 0.0f;
            bf16x8 pr;
            #pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(x[e] - base), p1 = __builtin_amdgcn_exp2f(x[e + 1] - base);
                sum += p0 + p1;
                const bf16x2 pp = __builtin_convertvector((f32x2){p0, p1}, bf16x2);
                pr[e] = pp[0];
                pr[e + 1] = pp[1];
            }
            l = l * fade + sum;
            if (__any(fade != 1.0f)) {
                #pragma unroll
                for (int c = 0; c < VB; ++c) acc[c] *= fade;
            }
            #pragma unroll
            for (int i = 0; i < VB / 4; ++i) {
                uint32_t a[4], b4[4];
                const uint32_t in0[4] = {v[0].w[i], v[1].w[i], v[2].w[i], v[3].w[i]};
                const uint32_t in1[4] = {v[4].w[i], v[5].w[i], v[6].w[i], v[7].w[i]};
                transpose4(in0, a);
                transpose4(in1, b4);
                #pragma unroll
                for (int c = 0; c < 4; ++c) {
                    bf16x8 vt;
                    decode4(a[c], v_scale, vt, 0);
                    decode4(b4[c], v_scale, vt, 4);
                    acc[4 * i + c] = dev::mma(vt, pr, acc[4 * i + c]);
                }
            }
            if (partial && __any(nan_seen)) {
                for (int t = 0; t < 32; ++t) {
                    if (r + t >= s.n) break;
                    #pragma unroll
                    for (int c = 0; c < VB; ++c)
                        #pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint8_t code = vb[(r + t) * rowb + h * D + (4 * g + j) * VB + c];
                            if ((code & 0x7F) == 0x7F && r + t <= pos) acc[c][j] = __builtin_nanf("");
                        }
                }
            }
        } else if (next >= 0) {
            load_k(next, k);
        }
        r = next;
    }

    // join the waves
    l = group_sum(l);
    if (g == 0) {
        ml_s[wave][li][0] = m;
        ml_s[wave][li][1] = l;
    }
    __syncthreads();
    float top = kNegInf, sum = 0.0f;
    #pragma unroll
    for (int i = 0; i < 4; ++i) top = __builtin_fmaxf(top, ml_s[i][li][0]);
    const float base = top == kNegInf ? 0.0f : top;
    #pragma unroll
    for (int i = 0; i < 4; ++i) sum += ml_s[i][li][1] * __builtin_amdgcn_exp2f(ml_s[i][li][0] - base);
    const float fade = __builtin_amdgcn_exp2f(m - base);
    #pragma unroll
    for (int j = 0; j < 4; ++j)
        #pragma unroll
        for (int c = 0; c < VB; c += 4)
            *reinterpret_cast<f32x4*>(&o_s[wave][li][(4 * g + j) * VB + c]) =
                (f32x4){acc[c][j] * fade, acc[c + 1][j] * fade, acc[c + 2][j] * fade, acc[c + 3][j] * fade};
    if (tid < 16) {  // wave 0: lane = row
        ml_s[0][li][0] = top;
        ml_s[0][li][1] = sum;
    }
    __syncthreads();
    const bool whole = s.nsplit == 1;
    const uint32_t slot = s.first_slot + w;
    constexpr int kPer = D / 4;  // threads of a row
    #pragma unroll
    for (int i = 0; i < 16 * kPer / kThreads; ++i) {
        const int rr = (i * kThreads + tid) / kPer, c = (tid % kPer) * 4;
        if (rr >= rows) continue;
        f32x4 o = *reinterpret_cast<const f32x4*>(&o_s[0][rr][c]);
        #pragma unroll
        for (int j = 1; j < 4; ++j) o += *reinterpret_cast<const f32x4*>(&o_s[j][rr][c]);
        if (!whole) {
            *reinterpret_cast<f32x4*>(p.part_o + ((int64_t)slot * 16 + rr) * D + c) = o;
            continue;
        }
        const float z = ml_s[0][rr][1], inv = z > 0.0f || z != z ? 1.0f / z : 0.0f;
        const int64_t tok = s.t0 + (SPARSE ? token : (r0 + rr) / G);
        const int64_t at = (tok * p.heads + (int64_t)h * G + (r0 + rr) % G) * D + c;
        const bf16x2 a = __builtin_convertvector((f32x2){o[0] * inv, o[1] * inv}, bf16x2);
        const bf16x2 b = __builtin_convertvector((f32x2){o[2] * inv, o[3] * inv}, bf16x2);
        *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.o) + at) =
            (u32x2){__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    }
    if (tid < rows) {
        const float mm = ml_s[0][tid][0], z = ml_s[0][tid][1];
        if (!whole) {
            *reinterpret_cast<f32x2*>(p.part_ml + ((int64_t)slot * 16 + tid) * 2) = (f32x2){mm, z};
        } else if (p.lse) {
            const int64_t tok = s.t0 + (SPARSE ? token : (r0 + tid) / G);
            p.lse[tok * p.heads + (int64_t)h * G + (r0 + tid) % G] = (mm + __builtin_amdgcn_logf(z)) * kLn2;
        }
    }
}

// Joins the runs of a tile: one workgroup for each output row.
template <int D>
__global__ __launch_bounds__(kThreads) void join_kernel(const KvbAttendParams p) {
    constexpr int kPer = D / 4, kWays = kThreads / kPer;
    __shared__ float o_s[kWays][D];
    const int64_t tok = blockIdx.x / (uint32_t)p.heads;
    const int head = (int)(blockIdx.x - tok * p.heads);
    int lo = 0, hi = p.n_seq - 1;  // last s with t0 <= tok
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.seq[mid].t0 <= tok) lo = mid; else hi = mid - 1;
    }
    const KvbAttendSeq& s = p.seq[__builtin_amdgcn_readfirstlane(lo)];
    if (s.nsplit == 1) return;
    const int G = p.heads / p.kv_heads, h = head / G;
    const int64_t t = tok - s.t0;
    int64_t item;
    int rr;
    if (p.idx) {
        item = (t * ((G + 15) / 16) + head % G / 16) * p.kv_heads + h;
        rr = head % G % 16;
    } else {
        const int64_t row = t * G + head % G;
        item = row / p.tile * p.kv_heads + h;
        rr = (int)(row % p.tile);
    }
    const int64_t slot = s.first_slot + item * s.nsplit;
    const float* ml = p.part_ml + (slot * p.tile + rr) * 2;
    const float* po = p.part_o + (slot * p.tile + rr) * D;
    float top = kNegInf;
    for (int i = 0; i < s.nsplit; ++i) top = __builtin_fmaxf(top, ml[(int64_t)i * p.tile * 2]);
    const float base = top == kNegInf ? 0.0f : top;
    const int tid = (int)threadIdx.x, way = tid / kPer, c = tid % kPer * 4;
    float sum = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = 0; i < s.nsplit; ++i) {
        const float f = __builtin_amdgcn_exp2f(ml[(int64_t)i * p.tile * 2] - base);
        sum += ml[(int64_t)i * p.tile * 2 + 1] * f;
        if (i % kWays == way) o += *reinterpret_cast<const f32x4*>(po + (int64_t)i * p.tile * D + c) * f;
    }
    *reinterpret_cast<f32x4*>(&o_s[way][c]) = o;
    __syncthreads();
    if (tid < kPer) {
        #pragma unroll
        for (int i = 1; i < kWays; ++i) o += *reinterpret_cast<const f32x4*>(&o_s[i][c]);
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
        const bf16x2 a = __builtin_convertvector((f32x2){o[0] * inv, o[1] * inv}, bf16x2);
        const bf16x2 b = __builtin_convertvector((f32x2){o[2] * inv, o[3] * inv}, bf16x2);
        *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.o) + ((int64_t)tok * p.heads + head) * D + c) =
            (u32x2){__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
        if (tid == 0 && p.lse) p.lse[tok * p.heads + head] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}

template <int D>
hipError_t launch(const KvbAttendParams& p, hipStream_t stream) {
    const void* fn = p.idx ? reinterpret_cast<const void*>(&attend_kernel<D, true>)
                           : reinterpret_cast<const void*>(&attend_kernel<D, false>);
    const hipError_t e = p.tile == 128 ? launch_kvb_prefill(p, stream) : launch_kernel(fn, dim3(p.wgs), dim3(kThreads), p, stream);
    if (e != hipSuccess || p.slots == 0) return e;
    return launch_kernel(reinterpret_cast<const void*>(&join_kernel<D>), dim3((uint32_t)(p.tokens * p.heads)), dim3(kThreads), p,
                         stream);
}

}  // namespace

hipError_t launch_kvb_attend(const KvbAttendParams& p, hipStream_t stream) {
    if (p.wgs == 0) return hipSuccess;
    return p.d == 64 ? launch<64>(p, stream) : p.d == 128 ? launch<128>(p, stream) : launch<256>(p, stream);
}

}  // namespace cap
