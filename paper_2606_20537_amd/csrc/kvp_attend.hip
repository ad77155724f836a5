// Causal attention of a step's tokens over a paged bf16 KV cache on gfx950.
//
//   x_j = scale q . k_j,  o = sum_j exp(x_j - m) v_j / l,  m = max x_j,
//   l = sum_j exp(x_j - m),  lse = m + log l,  over the rows j that the query
//   sees: max(0, pos - window + 1) <= j <= pos, on pages that are there
//
// in one pass over K and V with a running m and l.  The query rows of a KV head
// (tokens x query heads of the group) share its K and V: 16 of them are the
// columns of the matrix instructions, keys and channels the rows.
//  * S^T = K Q^T and O^T = V^T P^T on 16x16x32 bf16 tiles, sums in fp32.
//  * P goes in as two bf16 values, hi + lo, so that the weights keep 2^-16 and the
//    output's own rounding is the only one to 8 bits: the matrix pipes have nothing
//    else to do, as memory bounds the call.
// Both products leave a lane with one query row (lane % 16), so maximum, sum and
// correction need no value of another row, and S^T's accumulators are P^T's
// operand: lane group g holds keys 4g..4g+3 and 16+4g..16+4g+3 of 32, and loads
// V's rows in that order.  A lane reads 16 bytes of each of eight rows and transposes them
// in registers, two channels to a permute.  K and V go from memory to registers; LDS only
// joins the four waves, which take units of 32 rows in turn.
//
// Lengths and the table are read on the device, so that a captured call goes on with the
// sequences.  Every wave sums up the lengths for itself (a prefix sum over lanes) and
// finds the run of units that its workgroup takes: equal runs over all sequences, heads and
// tiles, so one long sequence beside many short ones spreads over the chip.  Segments that
// several workgroups share are joined by a second launch.
#include <hip/hip_runtime.h>

#include "device_util.h"
#include "kvp.h"

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
// Weights are 2^-24 of what exp(x - m) gives, so that sums of 2^24 values, the most that a
// sequence has, cannot overflow and means of finite values stay finite.
constexpr float kAbove = 24.0f;

__device__ inline float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }

// Maximum / sum over the four lanes that share lane % 16.
__device__ inline float group_max(float x) {
    x = __builtin_fmaxf(x, __shfl_xor(x, 16));
    return __builtin_fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float group_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// What scores are taken from, m the highest of them (-inf: none yet).
__device__ inline float reference(float m) { return m == kNegInf ? 0.0f : m + kAbove; }

// Inclusive prefix sum over the lanes of a wave (as dev::wave_inclusive_sum).
template <int CTRL, int ROW_MASK, bool BOUND_ZERO>
__device__ inline uint32_t dpp_u(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROW_MASK, 0xf, BOUND_ZERO);
}
__device__ inline uint32_t scan_lanes(uint32_t x) {
    x += dpp_u<0x111, 0xf, true>(x);
    x += dpp_u<0x112, 0xf, true>(x);
    x += dpp_u<0x114, 0xf, true>(x);
    x += dpp_u<0x118, 0xf, true>(x);
    x += dpp_u<0x142, 0xa, false>(x);
    x += dpp_u<0x143, 0xc, false>(x);
    return x;
}
__device__ inline int lane_int(int x, int l) { return __builtin_amdgcn_readlane(x, l); }
__device__ inline uint32_t lane_u32(uint32_t x, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); }

// What a wave's lane knows of sequence 64 chunk + lane.
struct Seq {
    int n, t0, T;      // rows held, first packed token, tokens
    int first, units;  // first unit, number of units (1 at least where T > 0)
    int tiles;         // of 16 query rows
    uint32_t weight;   // units of all its segments, with their beginnings
};

__device__ inline int clamp_token(const KvpAttendParams& p, int t) { return t < 0 ? 0 : t > p.tokens ? (int)p.tokens : t; }

__device__ inline Seq load_seq(const KvpAttendParams& p, int s) {
    const KvpPages& g = p.pages;
    Seq q = {};
    if (s >= g.n_seq) return q;
    q.n = g.lens[s];
    if (g.tok0) {
        q.t0 = clamp_token(p, g.tok0[s]);
        q.T = clamp_token(p, g.tok0[s + 1]) - q.t0;
    } else {
        q.t0 = s;
        q.T = s < p.tokens;
    }
    if (q.n < 0) q.n = 0;
    if (q.T <= 0) {
        q.T = 0;
        return q;
    }
    const int hi = q.n < g.capacity ? q.n : g.capacity;
    const int lo = p.window > 0 && q.n - q.T + 1 > p.window ? q.n - q.T + 1 - p.window : 0;
    q.first = lo / kKvpUnit;
    q.units = (hi + kKvpUnit - 1) / kKvpUnit - q.first;
    if (q.units < 1) q.units = 1;
    q.tiles = (int)(((int64_t)q.T * (p.heads / g.kv_heads) + 15) / 16);
    q.weight = (uint32_t)q.tiles * (uint32_t)g.kv_heads * (uint32_t)(q.units + kKvpBegin);
    return q;
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(const KvpAttendParams p) {
    constexpr int NJ = D / 32;                        // K: fragments of 32 channels
    constexpr int NV = D >= 128 ? D / 128 : 1;        // V: vectors of a lane
    constexpr int VC = D >= 128 ? 8 : 4;              // and their channels
    constexpr bool kAhead = D < 256;                  // registers for the next K beside V
    constexpr int kPitch = D + 4;
    __shared__ __attribute__((aligned(16))) float o_s[4][16][kPitch];
    __shared__ float ml_s[4][16][2], all_s[16][2];

    const KvpPages& g = p.pages;
    const int tid = (int)threadIdx.x, lane = tid & 63, li = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t w = blockIdx.x;
    const int G = p.heads / g.kv_heads;

    // the run [begin, end) of this workgroup
    const int chunks = (g.n_seq + 63) / 64;
    Seq q = load_seq(p, lane);
    uint32_t scan = scan_lanes(q.weight), before = 0;
    uint32_t total = lane_u32(scan, 63);
    for (int c = 1; c < chunks; ++c) total += lane_u32(scan_lanes(load_seq(p, 64 * c + lane).weight), 63);
    uint32_t per = (total + p.wgs - 1) / p.wgs;
    if (per < p.least) per = p.least;
    const uint32_t begin = w * per;
    if (begin >= total) return;
    const uint32_t end = begin + per < total ? begin + per : total;

    const int rowb = g.kv_heads * D * 2;
    uint32_t at = begin;  // where in the run we are
    int chunk = 0;
    bool again = false;   // LDS is in use
    while (at < end) {
        // the sequence that `at` is in (tok0 that does not ascend may make this fail: the run ends)
        while (at - before >= lane_u32(scan, 63)) {
            before += lane_u32(scan, 63);
            if (++chunk >= chunks) return;
            q = load_seq(p, 64 * chunk + lane);
            scan = scan_lanes(q.weight);
        }
        const int s = __builtin_popcountll(__ballot(scan <= at - before));
        if (s > 63) return;
        const int n = lane_int(q.n, s), seq_t0 = lane_int(q.t0, s), T = lane_int(q.T, s), units = lane_int(q.units, s);
        const uint32_t weight = lane_u32(q.weight, s), base = before + lane_u32(scan, s) - weight;
        const uint32_t size = (uint32_t)(units + kKvpBegin);
        if (at - base >= weight) return;
        const int segment = (int)((at - base) / size);
        const uint32_t seg0 = base + (uint32_t)segment * size;  // of the segment
        const uint32_t next = seg0 + size;
        const uint32_t unit0 = seg0 + kKvpBegin;                // of its first unit
        int u0 = 0, u1 = units;
        if (p.whole) {
            at = next;
            if (seg0 < begin) continue;  // its beginning was another workgroup's
        } else {
            u0 = at > unit0 ? (int)(at - unit0) : 0;
            u1 = end < next ? (int)(end - unit0) : units;
            at = next;
            if (u1 <= 0) continue;
        }
        const int tile = segment / g.kv_heads, h = segment - tile * g.kv_heads;
        const int first_unit = lane_int(q.first, s);
        const int seq = 64 * chunk + s;

        const int total_rows = T * G, r0 = tile * 16;
        const int rows = total_rows - r0 < 16 ? total_rows - r0 : 16;
        const int row = r0 + (li < rows ? li : rows - 1);  // rows past the last repeat it
        const int my_t = (int)((uint32_t)row / (uint32_t)G);
        const int pos = n - T + my_t;
        const int pos0 = n - T + (int)((uint32_t)r0 / (uint32_t)G), pos1 = n - T + (int)((uint32_t)(r0 + rows - 1) / (uint32_t)G);
        const int window = p.window > 0 ? p.window : 0x7fffffff;
        // keys above low are seen: pos - window, without passing 32 bits
        const int low = p.window > 0 ? (pos < 0 ? -1 : pos - window) : -1;
        const int low0 = p.window > 0 ? (pos0 < 0 ? -1 : pos0 - window) : -1, low1 = p.window > 0 ? (pos1 < 0 ? -1 : pos1 - window) : -1;

        // where 64 groups of 16 rows begin in the pools, a lane each; -1: on no page
        int64_t groups = -1;
        int group0 = 2 * (first_unit + u0);
        const int32_t* table = g.table + (int64_t)seq * g.table_stride;
        auto load_groups = [&]() {
            const uint32_t r = 16u * (uint32_t)(group0 + lane);
            groups = -1;
            if (r < (uint32_t)g.capacity && (int)r <= pos1) {
                const uint32_t column = r / (uint32_t)g.page;
                const int page = table[column];
                if ((uint32_t)page < (uint32_t)g.pages)
                    groups = (int64_t)page * g.page_stride + (int64_t)(r - column * (uint32_t)g.page) * rowb;
            }
        };
        auto group_at = [&](int i) -> int64_t {
            const uint32_t lo = (uint32_t)lane_int((int)(uint32_t)groups, i), hi = (uint32_t)lane_int((int)(groups >> 32), i);
            return (int64_t)((uint64_t)hi << 32 | lo);
        };
        load_groups();

        // the query rows, while the table is on its way
        bf16x8 qf[NJ];
        {
            const char* src = reinterpret_cast<const char*>(p.q.p) + (int64_t)(seq_t0 + my_t) * p.q.token +
                              (int64_t)(h * G + (row - my_t * G)) * p.q.head + 16 * grp;
            #pragma unroll
            for (int j = 0; j < NJ; ++j) qf[j] = *reinterpret_cast<const bf16x8*>(src + 64 * j);
        }

        f32x4 acc[NV * VC];
        #pragma unroll
        for (int c = 0; c < NV * VC; ++c) acc[c] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
        float m = kNegInf, l = 0.0f;

        u32x4 k[2][NJ];
        uint32_t v[8][NV * VC / 2];
        const int kvoff = li * rowb + h * D * 2 + 16 * grp, vvoff = 4 * grp * rowb + h * D * 2 + li * VC * 2;
        const char* kb = reinterpret_cast<const char*>(g.k);
        const char* vb = reinterpret_cast<const char*>(g.v);
        // (an absent group: nothing is read)
        auto load_k = [&](const int64_t (&a)[2]) {
            #pragma unroll
            for (int t = 0; t < 2; ++t) {
                const rsrc_t r = dev::make_rsrc_u32(kb + (a[t] < 0 ? 0 : a[t]), a[t] < 0 ? 0 : 16u * (uint32_t)rowb);
                #pragma unroll
                for (int j = 0; j < NJ; ++j) k[t][j] = __builtin_amdgcn_raw_buffer_load_b128(r, kvoff + 64 * j, 0, 0);
            }
        };
        auto load_v = [&](const int64_t (&a)[2]) {
            #pragma unroll
            for (int t = 0; t < 2; ++t) {
                const rsrc_t r = dev::make_rsrc_u32(vb + (a[t] < 0 ? 0 : a[t]), a[t] < 0 ? 0 : 16u * (uint32_t)rowb);
                #pragma unroll
                for (int e = 0; e < 4; ++e)
                    #pragma unroll
                    for (int x = 0; x < NV; ++x) {
                        if constexpr (VC == 8) {
                            const u32x4 d = __builtin_amdgcn_raw_buffer_load_b128(r, vvoff + 256 * x, e * rowb, 0);
                            #pragma unroll
                            for (int i = 0; i < 4; ++i) v[4 * t + e][4 * x + i] = d[i];
                        } else {
                            const u32x2 d = __builtin_amdgcn_raw_buffer_load_b64(r, vvoff, e * rowb, 0);
                            v[4 * t + e][0] = d[0];
                            v[4 * t + e][1] = d[1];
                        }
                    }
            }
        };

        // Groups of unit u (of the segment), those that the tile does not see as absent; waves move together
        // through the 64 groups that lanes hold.
        auto unit_groups = [&](int u, int64_t (&a)[2]) {
            const int r = (first_unit + u) * kKvpUnit;
            const bool seen = u < u1 && r <= pos1 && r + kKvpUnit - 1 > low0;
            #pragma unroll
            for (int t = 0; t < 2; ++t) a[t] = seen ? group_at(2 * (first_unit + u) + t - group0) : -1;
        };

        int64_t a[2];
        int u = u0 + wave;
        unit_groups(u, a);
        load_k(a);
        load_v(a);
        for (; u < u1; u += 4) {
            const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
            f32x4 s0 = zero, s1 = zero;
            #pragma unroll
            for (int j = 0; j < NJ; ++j) {
                s0 = dev::mma(__builtin_bit_cast(bf16x8, k[0][j]), qf[j], s0);
                s1 = dev::mma(__builtin_bit_cast(bf16x8, k[1][j]), qf[j], s1);
            }
            const int64_t now[2] = {a[0], a[1]};
            if (2 * (first_unit + u + 4) + 1 - group0 > 63) {
                group0 = 2 * (first_unit + u + 4);
                load_groups();
            }
            unit_groups(u + 4, a);
            if (kAhead) load_k(a);

            const int r = (first_unit + u) * kKvpUnit;
            float x[8];
            #pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = s0[e] * p.scale_log2;
                x[4 + e] = s1[e] * p.scale_log2;
            }
            const bool partial = r + kKvpUnit - 1 > pos0 || r <= low1 || now[0] < 0 || now[1] < 0;  // some row does not see every key
            bool bad = false;
            if (partial) {
                #pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int key = r + 4 * grp + (e < 4 ? e : 12 + e);
                    const bool there = now[e / 4] >= 0;
                    x[e] = there && key <= pos && key > low ? x[e] : kNegInf;
                    // a key that no row sees has no part in the product, whatever its V holds
                    const bool some = there && key <= pos1 && key > low0;
                    #pragma unroll
                    for (int i = 0; i < NV * VC / 2; ++i) {
                        uint32_t d = some ? v[e][i] : 0u;
                        // neither have infinities and NaN that some rows see and others do not: put back below
                        const uint32_t out = ((d & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((d & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
                        bad |= out != 0;
                        v[e][i] = d & ~out;
                    }
                }
            }
            float top = __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(x[0], x[1]), __builtin_fmaxf(x[2], x[3])),
                                        __builtin_fmaxf(__builtin_fmaxf(x[4], x[5]), __builtin_fmaxf(x[6], x[7])));
            top = __builtin_fmaxf(m, group_max(top));
            const float from = reference(top);
            const float fade = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(reference(m) - from);
            m = top;
            float sum = 0.0f, pf[8];
            bf16x8 hi, lo;
            #pragma unroll
            for (int e = 0; e < 8; ++e) {
                pf[e] = __builtin_amdgcn_exp2f(x[e] - from);
                sum += pf[e];
            }
            dev::split_n<8>(pf, hi, lo);
            l = l * fade + sum;
            if (__any(fade != 1.0f)) {
                #pragma unroll
                for (int c = 0; c < NV * VC; ++c) acc[c] *= fade;
            }
            #pragma unroll
            for (int i = 0; i < NV * VC / 2; ++i) {
                u32x4 even, odd;  // channels 2i and 2i + 1 of the eight keys
                #pragma unroll
                for (int e = 0; e < 4; ++e) {
                    even[e] = __builtin_amdgcn_perm(v[2 * e + 1][i], v[2 * e][i], 0x05040100u);
                    odd[e] = __builtin_amdgcn_perm(v[2 * e + 1][i], v[2 * e][i], 0x07060302u);
                }
                acc[2 * i] = dev::mma(__builtin_bit_cast(bf16x8, even), hi, acc[2 * i]);
                acc[2 * i + 1] = dev::mma(__builtin_bit_cast(bf16x8, odd), hi, acc[2 * i + 1]);
                acc[2 * i] = dev::mma(__builtin_bit_cast(bf16x8, even), lo, acc[2 * i]);
                acc[2 * i + 1] = dev::mma(__builtin_bit_cast(bf16x8, odd), lo, acc[2 * i + 1]);
            }
            if (partial && __any(bad)) {
                for (int t = 0; t < kKvpUnit; ++t) {
                    const int key = r + t;
                    const int64_t off = now[t / 16];
                    if (off < 0 || key > pos1 || key <= low0) continue;  // (uniform)
                    const int e = (t & 3) + (t >= 16 ? 4 : 0);
                    const float mine = e == 0 ? pf[0] : e == 1 ? pf[1] : e == 2 ? pf[2] : e == 3 ? pf[3] : e == 4 ? pf[4] : e == 5 ? pf[5] : e == 6 ? pf[6] : pf[7];
                    const float pk = __shfl(mine, li + 16 * (t % 16 / 4));
                    const uint16_t* src = reinterpret_cast<const uint16_t*>(vb + off + (int64_t)(t % 16) * rowb) + h * D;
                    #pragma unroll
                    for (int x = 0; x < NV; ++x)
                        #pragma unroll
                        for (int i = 0; i < VC; ++i)
                            #pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint32_t b = src[128 * x + VC * (4 * grp + j) + i];
                                if ((b & 0x7F80u) == 0x7F80u && key <= pos && key > low) acc[VC * x + i][j] += pk * bits_f32(b << 16);
                            }
                }
            }
            if (!kAhead) load_k(a);
            load_v(a);
        }

        // join the waves
        l = group_sum(l);
        if (again) __syncthreads();
        again = true;
        if (grp == 0) {
            ml_s[wave][li][0] = m;
            ml_s[wave][li][1] = l;
        }
        __syncthreads();
        float top = kNegInf, sum = 0.0f;
        #pragma unroll
        for (int i = 0; i < 4; ++i) top = __builtin_fmaxf(top, ml_s[i][li][0]);
        const float from = reference(top);
        #pragma unroll
        for (int i = 0; i < 4; ++i)
            sum += ml_s[i][li][0] == kNegInf ? ml_s[i][li][1] : ml_s[i][li][1] * __builtin_amdgcn_exp2f(reference(ml_s[i][li][0]) - from);
        const float fade = m == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(reference(m) - from);
        // (m is -inf where the wave saw nothing: zeros; or only NaN, which stays)
        #pragma unroll
        for (int x = 0; x < NV; ++x)
            #pragma unroll
            for (int j = 0; j < 4; ++j)
                #pragma unroll
                for (int i = 0; i < VC; i += 4)
                    *reinterpret_cast<f32x4*>(&o_s[wave][li][128 * x + VC * (4 * grp + j) + i]) =
                        (f32x4){acc[VC * x + i][j] * fade, acc[VC * x + i + 1][j] * fade, acc[VC * x + i + 2][j] * fade, acc[VC * x + i + 3][j] * fade};
        if (tid < 16) {  // wave 0: lane = row
            all_s[li][0] = top;
            all_s[li][1] = sum;
        }
        __syncthreads();
        // parts of the segment: the workgroups that have units of it
        const uint32_t from_wg = p.whole ? w : unit0 / per, parts = p.whole ? 1 : (next - 1) / per - from_wg + 1;
        const bool one = parts == 1;
        const uint32_t slot = 2 * w + (from_wg == w ? 1 : 0);
        constexpr int kPer = D / 4;  // threads of a row
        #pragma unroll
        for (int i = 0; i < 16 * kPer / kThreads; ++i) {
            const int rr = (i * kThreads + tid) / kPer, c = (tid % kPer) * 4;
            if (rr >= rows) continue;
            f32x4 o = *reinterpret_cast<const f32x4*>(&o_s[0][rr][c]);
            #pragma unroll
            for (int j = 1; j < 4; ++j) o += *reinterpret_cast<const f32x4*>(&o_s[j][rr][c]);
            if (!one) {
                *reinterpret_cast<f32x4*>(p.part_o + ((int64_t)slot * 16 + rr) * D + c) = o;
                continue;
            }
            const float z = all_s[rr][1], inv = z > 0.0f || z != z ? 1.0f / z : 0.0f;
            const int t = (int)((uint32_t)(r0 + rr) / (uint32_t)G);
            const int64_t to = ((int64_t)(seq_t0 + t) * p.heads + h * G + (r0 + rr - t * G)) * D + c;
            const bf16x2 lo2 = __builtin_convertvector((f32x2){o[0] * inv, o[1] * inv}, bf16x2);
            const bf16x2 hi2 = __builtin_convertvector((f32x2){o[2] * inv, o[3] * inv}, bf16x2);
            *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.o) + to) =
                (u32x2){__builtin_bit_cast(uint32_t, lo2), __builtin_bit_cast(uint32_t, hi2)};
        }
        if (tid < rows) {
            const float mm = all_s[tid][0], z = all_s[tid][1];
            const int t = (int)((uint32_t)(r0 + tid) / (uint32_t)G);
            const int64_t to = (int64_t)(seq_t0 + t) * p.heads + h * G + (r0 + tid - t * G);
            if (!one) *reinterpret_cast<f32x2*>(p.part_ml + ((int64_t)slot * 16 + tid) * 2) = (f32x2){mm, z};
            else if (p.lse) p.lse[to] = (reference(mm) + __builtin_amdgcn_logf(z)) * kLn2;
            if (!p.whole && from_wg == w) p.meta[to] = (uint64_t)tid << 48 | (uint64_t)parts << 24 | w;
        }
    }
}

// Joins the parts of a row: a workgroup has one output row, D / 4 threads to a part.
template <int D>
__global__ __launch_bounds__(kThreads) void join_kernel(const KvpAttendParams p) {
    constexpr int kPer = D / 4, kWays = kThreads / kPer;
    __shared__ __attribute__((aligned(16))) float o_s[kWays][D];
    __shared__ float ml_s[kWays][2];
    const KvpPages& g = p.pages;
    const int64_t out = (int64_t)blockIdx.y * kFp8GridX + blockIdx.x;
    if (out >= p.tokens * p.heads) return;
    const int tid = (int)threadIdx.x, way = tid / kPer, c = tid % kPer * 4;
    const uint64_t meta = p.meta[out];
    const int64_t token = out / p.heads;
    // a row that no sequence has: nothing was written for it
    const int64_t first = g.tok0 ? clamp_token(p, g.tok0[0]) : 0, last = g.tok0 ? clamp_token(p, g.tok0[g.n_seq]) : g.n_seq;
    if (token < first || token >= last) return;
    const int rr = (int)(meta >> 48) & 15;
    uint32_t parts = (uint32_t)(meta >> 24) & 0xFFFFFFu, w = (uint32_t)meta & 0xFFFFFFu;
    if (parts < 2 || w >= p.wgs || parts > p.wgs - w) return;
    float m = kNegInf, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t i = (uint32_t)way; i < parts; i += kWays) {
        const int64_t slot = 2 * (int64_t)(w + i) + (i == 0 ? 1 : 0);
        const f32x2 a = *reinterpret_cast<const f32x2*>(p.part_ml + (slot * 16 + rr) * 2);
        const f32x4 x = *reinterpret_cast<const f32x4*>(p.part_o + (slot * 16 + rr) * D + c);
        const float top = __builtin_fmaxf(m, a[0]), from = reference(top);
        const float f = m == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(reference(m) - from);
        const float e = a[0] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(reference(a[0]) - from);
        l = l * f + a[1] * e;
        o = o * f + x * e;
        m = top;
    }
    if (tid % kPer == 0) {
        ml_s[way][0] = m;
        ml_s[way][1] = l;
    }
    *reinterpret_cast<f32x4*>(&o_s[way][c]) = o;
    __syncthreads();
    if (way) return;
    m = kNegInf;
    l = 0.0f;
    o = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    #pragma unroll
    for (int i = 0; i < kWays; ++i) m = __builtin_fmaxf(m, ml_s[i][0]);
    #pragma unroll
    for (int i = 0; i < kWays; ++i) {
        const float e = ml_s[i][0] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(reference(ml_s[i][0]) - reference(m));
        l += ml_s[i][1] * e;
        o += *reinterpret_cast<const f32x4*>(&o_s[i][c]) * e;
    }
    const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
    const bf16x2 lo2 = __builtin_convertvector((f32x2){o[0] * inv, o[1] * inv}, bf16x2);
    const bf16x2 hi2 = __builtin_convertvector((f32x2){o[2] * inv, o[3] * inv}, bf16x2);
    *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.o) + out * D + c) =
        (u32x2){__builtin_bit_cast(uint32_t, lo2), __builtin_bit_cast(uint32_t, hi2)};
    if (c == 0 && p.lse) p.lse[out] = (reference(m) + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D>
hipError_t launch(const KvpAttendParams& p, hipStream_t stream) {
    void* args[] = {const_cast<KvpAttendParams*>(&p)};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&attend_kernel<D>), dim3(p.wgs), dim3(kThreads), args, 0, stream);
    if (e != hipSuccess || p.whole) return e;
    return hipLaunchKernel(reinterpret_cast<const void*>(&join_kernel<D>), wide_grid((uint64_t)(p.tokens * p.heads)), dim3(kThreads), args, 0, stream);
}

}  // namespace

hipError_t launch_kvp_attend(const KvpAttendParams& p, hipStream_t stream) {
    return p.d == 64 ? launch<64>(p, stream) : p.d == 128 ? launch<128>(p, stream) : launch<256>(p, stream);
}

}  // namespace cap
