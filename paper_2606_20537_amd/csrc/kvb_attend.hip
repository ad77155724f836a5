// Causal attention over a block-scaled FP8 KV cache on gfx950.
//
//   x_j = scale q . k_j,  o = sum_j exp(x_j - m) v_j / l,  m = max x_j,
//   l = sum_j exp(x_j - m),  lse = m + log l,  over the rows j that the query
//   sees (j <= its position; with a block list, of the listed blocks)
//
// in one pass over K and V with a running m and l.  The query rows of a KV head
// (tokens x query heads of the group) share its K and V: 16 of them are the
// columns of the matrix instructions, keys and channels the rows.
//  * S^T = K Q^T and O^T = V^T P^T on 16x16x32 bf16 tiles: the codes times their
//    power-of-two scale are exact in bf16.
//    The FP8 instructions would spare the conversion of K, but their sums lose what is
//    2^18 below a product of the same instruction (measured: up to 1.6e-4 of the sum of
//    the products' magnitudes, bf16 2e-7).
//  * P is rounded to bf16 (relative 2^-8 at most, as the output is); l sums the
//    unrounded P in 32 bits.
// Both products leave a lane with one query row (lane % 16), so maximum, sum and
// correction need no value of another row, and S^T's accumulators are P^T's
// operand: lane group g holds keys 4g..4g+3 and 16+4g..16+4g+3 of 32, and loads
// V's rows in that order.  A lane reads d / 16 contiguous bytes of eight rows and
// transposes them in registers.  K and V go from memory to registers; LDS only
// joins the four waves, which take 32 rows of the cache in turn.
//
// What bounds it, 8 query heads on each KV head of 256 channels, one token: 131072 +
// 18561 rows, 307 MB, 58.2 us (5.3 TB/s, the rate of a copy); 16385 rows, 33.8 MB, 10.8 us
// and 4.5 of the join, of which the data take 6.5 and the launches 2.2 each.  A wave
// takes about 1 us for 32 rows by itself (128 byte permutes and conversions, 32 matrix
// instructions, little of it side by side), so runs stay a few blocks long.  Registers for
// V of a second unit pay up to 128 channels; at 256 they spill.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "kvb_device.h"

namespace cap {
namespace {

using dev::bf16x8;
using dev::f32x4;
using dev::rsrc_t;
using dev::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr float kNegInf = -__builtin_inff();
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLargeV = 0x1p87f;  // a scale: codes are below 2^9

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

// 16 keys (lane % 16: a key, chunk j of 16 bytes: channels 64 j + 16 g .. + 15) against the
// query rows, whose channels a lane holds in the same order.
template <int D>
__device__ inline f32x4 scores(const u32x4* k, float scale, const bf16x8* q) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    #pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        bf16x8 a;
        decode4(k[j / 2][2 * (j % 2)], scale, a, 0);
        decode4(k[j / 2][2 * (j % 2) + 1], scale, a, 4);
        s = dev::mma(a, q[j], s);
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

template <int D, bool SPARSE, int N>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(const KvbAttendTable<N> p) {
    constexpr int VB = D / 16, NJ = D / 64;
    constexpr bool kAhead = D < 256;  // registers for V of two units
    constexpr int kPitch = D + 4;
    __shared__ float o_s[4][16][kPitch];
    __shared__ float ml_s[4][16][2], all_s[16][2];

    const uint32_t block = kvb_block();
    if (block >= p.wgs) return;
    const KvbAttendSeq& s = p.seq[KVB_SEQ_OF(p, first_wg, block)];
    const uint32_t w = block - s.first_wg;
    const int G = p.heads / p.kv_heads;
    const uint32_t item = w / (uint32_t)s.nsplit;  // (tile, kv head)
    const int split = (int)(w - item * (uint32_t)s.nsplit);
    const int h = (int)(item % (uint32_t)p.kv_heads);
    int64_t tile = item / (uint32_t)p.kv_heads;
    // the tile's rows: `rows` of them from row r0 of the sequence, or of token `token` (sparse)
    int64_t r0, total;
    int64_t token = 0;
    if (SPARSE) {
        const int per = (G + 15) / 16;
        token = row_div(tile, per);
        r0 = (tile - token * per) * 16;
        total = G;
    } else {
        total = (int64_t)s.T * G;
        tile = (total + 15) / 16 - 1 - tile;  // the longest first
        r0 = tile * 16;
    }
    const int rows = (int)(total - r0 < 16 ? total - r0 : 16);
    const int tid = (int)threadIdx.x, lane = tid & 63, li = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row = r0 + (li < rows ? li : rows - 1);  // rows past the last repeat it
    const int64_t my_token = SPARSE ? token : row_div(row, G);
    const int64_t pos = s.n - s.T + my_token;              // the last key that the row sees
    const int64_t pos0 = s.n - s.T + (SPARSE ? token : row_div(r0, G)), pos1 = s.n - s.T + (SPARSE ? token : row_div(r0 + rows - 1, G));

    const int rowb = p.kv_heads * D;
    const uint8_t* kb = reinterpret_cast<const uint8_t*>(s.k);
    const uint8_t* vb = reinterpret_cast<const uint8_t*>(s.v);
    const global_ptr<float> sc = (global_ptr<float>)s.scales;
    const int kvoff = li * rowb + h * D + 16 * g, vvoff = 4 * g * rowb + h * D + li * VB;
    const int32_t* list = SPARSE ? p.idx + ((s.t0 + token) * p.kv_heads + h) * p.n_sel : nullptr;

    const int nblk = SPARSE ? p.n_sel : tile_blocks(s, r0, 16, total, G), runs = tile_runs(s, nblk);
    if (split >= runs) return;
    const int begin = split * s.per, end = begin + s.per < nblk ? begin + s.per : nblk;
    const int units = 2 * (end - begin);

    // the run's list entries, one to a lane (kKvbListRun at most)
    int entries = -1;
    if (SPARSE && begin + lane < end) entries = list[begin + lane];
    // first row of unit u (32 rows); -1: nothing there (an entry that names no visible block)
    auto unit_row = [&](int u) -> int64_t {
        if (u >= units) return -1;
        int64_t b = begin + (u >> 1);
        if (SPARSE) {
            b = __builtin_amdgcn_readlane(entries, u >> 1);
            if (b < 0 || b * kKvbBlock > pos) return -1;
        }
        const int64_t r = b * kKvbBlock + 32 * (u & 1);
        return r <= pos1 ? r : -1;
    };
    auto load_k = [&](int64_t r, u32x4 (&k)[2][NJ]) {
        const rsrc_t rk = dev::make_rsrc_u32(kb + (r < 0 ? 0 : r) * rowb, r < 0 ? 0 : 32u * rowb);  // r < 0: nothing is read
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

    auto load_values = [&](int64_t r, VBytes<VB> (&v)[8]) {
        const rsrc_t rv = dev::make_rsrc_u32(vb + (r < 0 ? 0 : r) * rowb, r < 0 ? 0 : 32u * rowb);
        #pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = load_v<VB>(rv, vvoff, (e < 4 ? e : 12 + e) * rowb);
    };
    // The scales of a unit are loaded ahead of its K (loads return in order), K once the K
    // before it is used, V at the start of the step before the unit's own (or of its own).  With
    // 256 channels the scales go two steps ahead, as K waits for its own (16385 rows 13.4 us
    // a pass, one step ahead 13.8; of 128 channels, 6 tokens at 16390, 15.3 and 14.9).
    u32x4 k[2][NJ];
    VBytes<VB> v[kAhead ? 2 : 1][8];
    float scales[2], ahead[2];
    auto load_scales = [&](int64_t r, float (&scales)[2]) {
        const int64_t b = r < 0 ? 0 : r / kKvbBlock;
        scales[0] = sc[(b * 2) * p.kv_heads + h];
        scales[1] = sc[(b * 2 + 1) * p.kv_heads + h];
    };
    int64_t r = unit_row(wave);
    load_scales(r, scales);
    if (!kAhead) load_scales(unit_row(wave + 4), ahead);
    load_k(r, k);
    if (kAhead) load_values(r, v[0]);
    // the query rows, while the first keys are on their way
    bf16x8 q[D / 32];
    {
        const uint8_t* src = static_cast<const uint8_t*>(p.q) + (s.t0 + my_token) * p.q_stride + ((int64_t)h * G + row_mod(row, G)) * D * 2;
        #pragma unroll
        for (int j = 0; j < D / 32; ++j) q[j] = *reinterpret_cast<const bf16x8*>(src + (64 * (j / 2) + 16 * g + 8 * (j % 2)) * 2);
    }

    auto step = [&](int u, VBytes<VB> (&vc)[8], VBytes<VB> (&vn)[8]) {
        const int64_t next = unit_row(u + 4);
        if (kAhead) load_values(next, vn); else load_values(r, vc);
        const float k_scale = scales[0], v_scale = scales[1];
        const f32x4 s0 = scores<D>(k[0], k_scale, q), s1 = scores<D>(k[1], k_scale, q);
        if (kAhead) {
            load_scales(next, scales);
        } else {
            scales[0] = ahead[0];
            scales[1] = ahead[1];
            load_scales(unit_row(u + 8), ahead);
        }
        load_k(next, k);
        const int64_t now = r;
        r = next;
        if (now < 0) return;
        float x[8];
        #pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = s0[e] * p.scale_log2;
            x[4 + e] = s1[e] * p.scale_log2;
        }
        const bool partial = now + 31 > pos0;  // some row does not see every key
        uint32_t nan_seen = 0;
        if (partial) {
            // of the unit's rows: the last that the query row sees, and how many there are
            const int sees = (int)(pos - now < 32 ? pos - now : 32), held = (int)(s.n - now < 32 ? s.n - now : 32);
            #pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = 4 * g + (e < 4 ? e : 12 + e);
                x[e] = key > sees ? kNegInf : x[e];
                const uint32_t there = key < held ? ~0u : 0u;
                // NaN in V times a weight of zero would be NaN: such codes go, and are put back below
                #pragma unroll
                for (int i = 0; i < VB / 4; ++i) {
                    const uint32_t bad = nan_bytes(vc[e].w[i]);
                    nan_seen |= bad & there;
                    vc[e].w[i] &= ~(bad | (bad - (bad >> 7)));
                }
            }
        }
        float top = __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(x[0], x[1]), __builtin_fmaxf(x[2], x[3])),
                                    __builtin_fmaxf(__builtin_fmaxf(x[4], x[5]), __builtin_fmaxf(x[6], x[7])));
        // Sums of 2^31 values of 2^96 would overflow: beside such blocks the reference stands 2^32
        // above the highest score, with weights of 2^-32 (any reference will do, as long as O and l share it).
        top = __builtin_fmaxf(m, group_max(top) + (v_scale > kLargeV ? 32.0f : 0.0f));
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
            const uint32_t in0[4] = {vc[0].w[i], vc[1].w[i], vc[2].w[i], vc[3].w[i]};
            const uint32_t in1[4] = {vc[4].w[i], vc[5].w[i], vc[6].w[i], vc[7].w[i]};
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
        if (partial && __any(nan_seen != 0)) {
            for (int t = 0; t < 32; ++t) {
                if (now + t >= s.n) break;
                #pragma unroll
                for (int c = 0; c < VB; ++c)
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint8_t code = vb[(now + t) * rowb + h * D + (4 * g + j) * VB + c];
                        if ((code & 0x7F) == 0x7F && now + t <= pos) acc[c][j] = __builtin_nanf("");
                    }
            }
        }
    };
    for (int u = wave; u < units; u += 8) {
        step(u, v[0], v[kAhead ? 1 : 0]);
        if (u + 4 < units) step(u + 4, v[kAhead ? 1 : 0], v[0]);
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
        all_s[li][0] = top;
        all_s[li][1] = sum;
    }
    __syncthreads();
    const bool whole = runs == 1;
    const uint32_t slot = s.first_slot + (uint32_t)((tile * p.kv_heads + h) * s.nsplit + split);
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
        const float z = all_s[rr][1], inv = z > 0.0f || z != z ? 1.0f / z : 0.0f;
        const int64_t tok = s.t0 + (SPARSE ? token : row_div(r0 + rr, G));
        const int64_t at = (tok * p.heads + (int64_t)h * G + row_mod(r0 + rr, G)) * D + c;
        const bf16x2 a = __builtin_convertvector((f32x2){o[0] * inv, o[1] * inv}, bf16x2);
        const bf16x2 b = __builtin_convertvector((f32x2){o[2] * inv, o[3] * inv}, bf16x2);
        *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.o) + at) =
            (u32x2){__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    }
    if (tid < rows) {
        const float mm = all_s[tid][0], z = all_s[tid][1];
        if (!whole) {
            *reinterpret_cast<f32x2*>(p.part_ml + ((int64_t)slot * 16 + tid) * 2) = (f32x2){mm, z};
        } else if (p.lse) {
            const int64_t tok = s.t0 + (SPARSE ? token : row_div(r0 + tid, G));
            p.lse[tok * p.heads + (int64_t)h * G + row_mod(r0 + tid, G)] = (mm + __builtin_amdgcn_logf(z)) * kLn2;
        }
    }
}

// Joins the runs of a tile.  A thread takes 16 bytes of an output row; with WAYS > 1,
// for many runs, a workgroup has 64 channels of one row and WAYS threads share the
// runs of each 16 bytes.
template <int D, int WAYS, int N>
__global__ __launch_bounds__(kThreads) void join_kernel(const KvbAttendTable<N> p) {
    constexpr int kPer = WAYS > 1 ? kThreads / WAYS : D / 4, kRows = kThreads / kPer / WAYS, kParts = WAYS > 1 ? D / (4 * kPer) : 1;
    constexpr int kAhead = 4;  // runs whose loads are in flight
    static_assert(kPer * kParts == D / 4 && kRows * kPer * WAYS == kThreads, "threads of a row");
    const int tid = (int)threadIdx.x, way = tid / kPer % WAYS, mine = tid / (kPer * WAYS);
    const uint32_t block = kvb_block();
    const int c = (int)(block % kParts) * 4 * kPer + tid % kPer * 4;
    const uint32_t all = (uint32_t)(p.tokens * p.heads), out = block / kParts * kRows + (uint32_t)mine;
    const uint32_t at = out < all ? out : all - 1;  // threads past the last row repeat it
    const uint32_t tok = at / (uint32_t)p.heads;
    const int head = (int)(at - tok * (uint32_t)p.heads);
    int seq = 0;
    if (WAYS > 1) {
        seq = KVB_SEQ_OF(p, t0, (int64_t)tok);
    } else {
        int hi = p.n_seq - 1;  // last s with t0 <= tok
        while (seq < hi) {
            const int mid = (seq + hi + 1) >> 1;
            if (p.seq[mid].t0 <= (int64_t)tok) seq = mid; else hi = mid - 1;
        }
    }
    seq = seq < 0 ? 0 : seq;
    const KvbAttendSeq& s = p.seq[seq];
    const int G = p.heads / p.kv_heads, h = head / G;
    const int64_t t = (int64_t)tok - s.t0;
    int64_t item;
    int rr, n = 1;  // one run: written by its workgroup (or by another launch), nothing to do
    if (p.idx) {
        item = (t * ((G + 15) / 16) + head % G / 16) * p.kv_heads + h;
        rr = head % G % 16;
        n = s.nsplit;
    } else {
        const int64_t row = t * G + head % G;
        item = (int64_t)row_div(row, p.tile) * p.kv_heads + h;
        rr = (int)row_mod(row, p.tile);
        if (t >= 0 && t < s.T) n = tile_runs(s, tile_blocks(s, row - rr, p.tile, (int64_t)s.T * G, G));
    }
    const int64_t slot = s.first_slot + item * s.nsplit;
    const global_ptr<f32x2> ml = (global_ptr<f32x2>)(p.part_ml + (slot * p.tile + rr) * 2);
    const global_ptr<f32x4> po = (global_ptr<f32x4>)(p.part_o + (slot * p.tile + rr) * D + c);
    const int ml_step = p.tile, po_step = p.tile * D / 4;
    float top = kNegInf, sum = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = way; n > 1 && i < n; i += kAhead * WAYS) {
        f32x2 a[kAhead];
        f32x4 x[kAhead];
        #pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int j = i + k * WAYS < n ? i + k * WAYS : i;
            a[k] = ml[(int64_t)j * ml_step];
            x[k] = po[(int64_t)j * po_step];
        }
        #pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i + k * WAYS >= n) continue;
            const float up = __builtin_fmaxf(top, a[k][0]), base = up == kNegInf ? 0.0f : up;
            const float f = __builtin_amdgcn_exp2f(top - base), g = __builtin_amdgcn_exp2f(a[k][0] - base);
            sum = sum * f + a[k][1] * g;
            o = o * f + x[k] * g;
            top = up;
        }
    }
    if constexpr (WAYS > 1) {
        __shared__ float o_s[WAYS - 1][4 * kPer], ml_s[WAYS][2];
        if (tid % kPer == 0) {
            ml_s[way][0] = top;
            ml_s[way][1] = sum;
        }
        __syncthreads();
        float up = kNegInf;
        #pragma unroll
        for (int i = 0; i < WAYS; ++i) up = __builtin_fmaxf(up, ml_s[i][0]);
        const float base = up == kNegInf ? 0.0f : up;
        sum = 0.0f;
        #pragma unroll
        for (int i = 0; i < WAYS; ++i) sum += ml_s[i][1] * __builtin_amdgcn_exp2f(ml_s[i][0] - base);
        o *= __builtin_amdgcn_exp2f(top - base);
        top = up;
        if (way) *reinterpret_cast<f32x4*>(&o_s[way - 1][tid % kPer * 4]) = o;
        __syncthreads();
        if (way) return;
        #pragma unroll
        for (int i = 1; i < WAYS; ++i) o += *reinterpret_cast<const f32x4*>(&o_s[i - 1][tid % kPer * 4]);
    }
    if (n == 1 || out >= all) return;
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    const bf16x2 a = __builtin_convertvector((f32x2){o[0] * inv, o[1] * inv}, bf16x2);
    const bf16x2 b = __builtin_convertvector((f32x2){o[2] * inv, o[3] * inv}, bf16x2);
    *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.o) + (int64_t)out * D + c) =
        (u32x2){__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    if (c == 0 && p.lse) p.lse[out] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

#define KVB_FORMS(kernel, ...) reinterpret_cast<const void*>(&kernel<__VA_ARGS__, kKvbFew>), reinterpret_cast<const void*>(&kernel<__VA_ARGS__, KVB_MAX_SEQ>)

template <int D>
hipError_t launch(const KvbAttendParams& p, hipStream_t stream) {
    const dim3 block(kThreads);
    const hipError_t e = p.tile == 128 ? launch_kvb_prefill(p, stream)
                         : p.idx ? launch_kvb<KvbAttendTable>(KVB_FORMS(attend_kernel, D, true), kvb_grid(p.wgs), block, p, stream)
                                 : launch_kvb<KvbAttendTable>(KVB_FORMS(attend_kernel, D, false), kvb_grid(p.wgs), block, p, stream);
    if (e != hipSuccess || p.slots == 0) return e;
    // Threads side by side on the runs of a row where there are few rows for the chip: 161 tokens x
    // 32 heads x 256 channels of 8 runs took 30 us with them, 32 heads of one token and 43 runs 10 us without.
    const uint32_t rows = (uint32_t)(p.tokens * p.heads), per = kThreads / (D / 4);
    int runs = 0;
    for (int i = 0; i < p.n_seq; ++i) runs = p.seq[i].nsplit > runs ? p.seq[i].nsplit : runs;
    return runs > 4 && rows * (D / 64) <= 4096
               ? launch_kvb<KvbAttendTable>(KVB_FORMS(join_kernel, D, 16), kvb_grid(rows * (D / 64)), block, p, stream)
               : launch_kvb<KvbAttendTable>(KVB_FORMS(join_kernel, D, 1), kvb_grid((rows + per - 1) / per), block, p, stream);
}

}  // namespace

hipError_t launch_kvb_attend(const KvbAttendParams& p, hipStream_t stream) {
    if (p.wgs == 0) return hipSuccess;
    return p.d == 64 ? launch<64>(p, stream) : p.d == 128 ? launch<128>(p, stream) : launch<256>(p, stream);
}

}  // namespace cap
