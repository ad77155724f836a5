// Causal attention of a step's tokens over a paged bf16 KV cache on gfx950.
//
//   x_j = scale q . k_j,  o = sum_j exp(x_j - m) v_j / l,  m = max x_j,
//   l = sum_j exp(x_j - m),  lse = m + log l,  over the rows j that the query
//   sees: max(0, pos - window + 1) <= j <= pos, on pages that are there
//
// in one pass over K and V with a running m (or one a little below the maximum) and l.  The query rows of a KV head
// (tokens x query heads of the group) share its K and V: 16 of them, twice 16 or eight times, are the
// columns of the matrix instructions, keys and channels the rows.
//  * S^T = K Q^T and O^T = V^T P^T on 16x16x32 bf16 tiles, sums in fp32.
//  * P goes in as three bf16 values, in which the weights keep fp32's 24 bits: memory
//    bounds the call, and the matrix pipes are 9 % busy.  In tiles of 128 rows, which arithmetic
//    bounds, they are two, and the weights keep 2^-16, so that the output's own rounding stays the largest: 16384 tokens, 32 heads on 4
//    of 64, 128 and 256 channels 2.43, 3.62 and 7.93 ms, with three 3.05, 4.46 and 9.30.
// Both products leave a lane with one query row (lane % 16), so maximum, sum and
// correction need no value of another row, and S^T's accumulators are P^T's
// operand: lane group g holds keys 4g..4g+3 and 16+4g..16+4g+3 of 32, in which order the
// transposing reads of LDS give V's.
//
// A wave takes units of 32 rows.  K and V go from memory to LDS without registers, to a slot of
// each that no other wave uses, so the waves wait for their own loads and never for each other;
// the next K is on its way once a K has been read, the next V likewise.  That keeps 96 to 128 KiB on
// their way to each CU.  With both in registers 64 to 128 KiB would fit, but the compiler,
// which cannot tell the loads apart, waited for all of them at every step: 4.6 to 5.5 TB/s
// over 1 GB, now 5.9 to 6.2 (and 6.8 over 4.3 GB).  Loads are streamed: cached ones read 1 GB 12 % slower, and
// what fits the last cache 7 % faster, which a stack of layers does not.
//
// Lengths and the table are read on the device, so that a captured call goes on with the
// sequences.  Every wave sums up the lengths for itself (a prefix sum over lanes) and
// finds the units that its workgroup takes: even parts of segments, or where there is more work equal
// runs over all sequences, heads and tiles, so that one long sequence beside many short ones spreads
// over the chip.  Segments that several workgroups share are joined by a second launch.
//
// Long runs of tokens (prompts, resumed turns) have tiles of 128 query rows, where arithmetic counts: each wave
// has its own rows and all of the units, which the waves load together into a ring of four, with
// a barrier to each, so that K and V come from memory once for 128 rows and not for 32.  16384 tokens behind none, 32 heads on 4 of
// 64, 128 and 256 channels: 2.4, 3.6 and 8.0 ms (floor 0.9, 1.8, 3.6; in tiles of 32 rows 5.8, 11.3, 26.1): 0.67 to 0.91 PFLOP/s
// of matrix instructions with both parts of P, and between them the weights' exponentials.  Loads are kept by the caches here, as other tiles read the same.
//
// What bounds it, one token, 8 query heads on each KV head of 256 channels: 131072 + 16449 + 2111 + 1 rows
// x 4 heads, 613 MB, 100 us + 5 of the join (6.1 TB/s); 16385 rows x 4, 67 MB, 18 + 4, of which the data take
// 10, the way to the first load 4 (lengths, table and 400 instructions behind each other) and the last sums 2.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "device_util.h"
#include "kvp.h"

namespace cap {
namespace {

using dev::bf16x8;
using dev::f32x4;
using dev::u32x4;
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr float kNegInf = -__builtin_inff();
constexpr float kLn2 = 0.6931471805599453f;
// m may stay up to kBehind below the highest score so far (log2 units), as a new m has all rows' sums multiplied, and comes
// seldom so: 512 tokens of 16 sequences, 16 heads on 4 of 64 and 256 channels 209 and 556 us with every new one, 193 and 512 so.
// Sums of large values may leave fp32's range where their mean does not.  Such segments are taken a second time, with weights
// of 2^-kAbove of what exp(x - m) gives, 2^-24 at most, so that sums of 2^24 values, the most that a sequence has, stay finite; and only
// means that were not finite are replaced, as small values in other channels would lose bits to such weights.
constexpr float kBehind = 8.0f, kAbove = 24.0f + kBehind;
// Parts of even cuts at least (a unit to each wave) and at most; with longer ones equal runs leave fewer workgroups idle.
constexpr uint32_t kLeastCut = 4, kMostCut = 32;

typedef const char __attribute__((address_space(1)))* global_bytes;
typedef __attribute__((address_space(3))) char* lds_bytes;
typedef const void __attribute__((address_space(1)))* lds_source;
typedef __attribute__((address_space(3))) void* lds_target;
// Reads of what load_lds has brought, which wait for their answers themselves.  (Before its own reads of LDS the compiler
// would wait for every load on its way.)
// 16 bytes at `at` and `more` behind it, for four addresses.
template <int MORE>
__device__ inline void read_k4(const uint32_t (&at)[4], u32x4 (&x)[8]) {
    asm volatile(
        "ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:%12\n\t"
        "ds_read_b128 %2, %9\n\tds_read_b128 %3, %9 offset:%12\n\t"
        "ds_read_b128 %4, %10\n\tds_read_b128 %5, %10 offset:%12\n\t"
        "ds_read_b128 %6, %11\n\tds_read_b128 %7, %11 offset:%12\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "i"(MORE)
        : "memory");
}
template <int MORE>
__device__ inline void read_k2(const uint32_t (&at)[2], u32x4 (&x)[4]) {
    asm volatile(
        "ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:%6\n\t"
        "ds_read_b128 %2, %5\n\tds_read_b128 %3, %5 offset:%6\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
        : "v"(at[0]), "v"(at[1]), "i"(MORE)
        : "memory");
}
template <int MORE>
__device__ inline void read_k8(const uint32_t (&at)[8], u32x4 (&x)[16]) {
    asm volatile(
        "ds_read_b128 %0, %16\n\tds_read_b128 %1, %16 offset:%24\n\t"
        "ds_read_b128 %2, %17\n\tds_read_b128 %3, %17 offset:%24\n\t"
        "ds_read_b128 %4, %18\n\tds_read_b128 %5, %18 offset:%24\n\t"
        "ds_read_b128 %6, %19\n\tds_read_b128 %7, %19 offset:%24\n\t"
        "ds_read_b128 %8, %20\n\tds_read_b128 %9, %20 offset:%24\n\t"
        "ds_read_b128 %10, %21\n\tds_read_b128 %11, %21 offset:%24\n\t"
        "ds_read_b128 %12, %22\n\tds_read_b128 %13, %22 offset:%24\n\t"
        "ds_read_b128 %14, %23\n\tds_read_b128 %15, %23 offset:%24\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7]), "=&v"(x[8]), "=&v"(x[9]),
          "=&v"(x[10]), "=&v"(x[11]), "=&v"(x[12]), "=&v"(x[13]), "=&v"(x[14]), "=&v"(x[15])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]), "v"(at[7]), "i"(MORE)
        : "memory");
}
// N words (4 or 8).
template <int N>
__device__ inline void read_words(uint32_t at, u32x4 (&x)[2]) {
    if constexpr (N == 4) asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(x[0]) : "v"(at) : "memory");
    else asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:16\n\ts_waitcnt lgkmcnt(0)" : "=&v"(x[0]), "=&v"(x[1]) : "v"(at) : "memory");
}
// Transposing reads of bf16 rows: lane n of 16 gets four rows of channel n, at `at` and `more` behind it.
template <int MORE>
__device__ inline void read_v4(const uint32_t (&at)[4], u32x2 (&x)[8]) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
        "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
        "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
        "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "i"(MORE)
        : "memory");
}
template <int MORE>
__device__ inline void read_v8(const uint32_t (&at)[8], u32x2 (&x)[16]) {
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16\n\tds_read_b64_tr_b16 %1, %16 offset:%24\n\t"
        "ds_read_b64_tr_b16 %2, %17\n\tds_read_b64_tr_b16 %3, %17 offset:%24\n\t"
        "ds_read_b64_tr_b16 %4, %18\n\tds_read_b64_tr_b16 %5, %18 offset:%24\n\t"
        "ds_read_b64_tr_b16 %6, %19\n\tds_read_b64_tr_b16 %7, %19 offset:%24\n\t"
        "ds_read_b64_tr_b16 %8, %20\n\tds_read_b64_tr_b16 %9, %20 offset:%24\n\t"
        "ds_read_b64_tr_b16 %10, %21\n\tds_read_b64_tr_b16 %11, %21 offset:%24\n\t"
        "ds_read_b64_tr_b16 %12, %22\n\tds_read_b64_tr_b16 %13, %22 offset:%24\n\t"
        "ds_read_b64_tr_b16 %14, %23\n\tds_read_b64_tr_b16 %15, %23 offset:%24\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7]), "=&v"(x[8]), "=&v"(x[9]), "=&v"(x[10]), "=&v"(x[11]), "=&v"(x[12]), "=&v"(x[13]), "=&v"(x[14]), "=&v"(x[15])
        : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]), "v"(at[7]), "i"(MORE)
        : "memory");
}
// 1 KiB into LDS, 16 bytes from each lane's address; streamed, or kept for the tiles that read it again.
template <bool STREAM>
__device__ inline void load_lds(global_bytes from, lds_bytes to) {
    if constexpr (STREAM) __builtin_amdgcn_global_load_lds((lds_source)from, (lds_target)to, 16, 0, 2);
    else __builtin_amdgcn_global_load_lds((lds_source)from, (lds_target)to, 16, 0, 0);
}
// What a row's number changes in the places of its pieces: rows that lie over the same banks differ.
template <int D>
__device__ constexpr int fold_k(int row) { return D == 64 ? row >> 1 & 7 : row & 15; }
template <int D>
__device__ constexpr int fold_v(int row) { return D == 256 ? row & 15 : D == 128 ? row & 7 : row >> 1 & 3; }
// The same value, of which the compiler does not know that it stays the same: what is derived from it is not
// kept in registers over a loop.
template <class T>
__device__ inline T hidden(T x) {
    asm volatile("" : "+v"(x));
    return x;
}
// The kernel's arguments, to be read where they are used instead of being held from the kernel's beginning.
template <class T>
__device__ inline const T* hidden_arguments() {
    auto at = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return (const T*)at;
}
// Until at most N loads of this wave are on their way (they come in order).
template <int N>
__device__ inline void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}
// Until this wave's reads of LDS have been answered.
__device__ inline void wait_lds() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ inline float bits_f32(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ inline uint32_t f32_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

// x of the lanes in even rows of 16 and of those in odd ones, or of the lower and of the upper 32 lanes, each in both.
__device__ inline f32x2 both16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(f32_bits(x), f32_bits(x), false, false);
    return (f32x2){bits_f32(r[0]), bits_f32(r[1])};
}
__device__ inline f32x2 both32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(f32_bits(x), f32_bits(x), false, false);
    return (f32x2){bits_f32(r[0]), bits_f32(r[1])};
}
// Maximum / sum over the four lanes that share lane % 16.
__device__ inline float group_max(float x) {
    const f32x2 a = both16(x), b = both32(__builtin_fmaxf(a[0], a[1]));
    return __builtin_fmaxf(b[0], b[1]);
}
__device__ inline float group_sum(float x) {
    const f32x2 a = both16(x), b = both32(a[0] + a[1]);
    return b[0] + b[1];
}
// Four values times f, rounded to bf16.
__device__ inline u32x2 bf16x4_of(const f32x4& o, float f) {
    const bf16x2 lo = __builtin_convertvector((f32x2){o[0] * f, o[1] * f}, bf16x2);
    const bf16x2 hi = __builtin_convertvector((f32x2){o[2] * f, o[3] * f}, bf16x2);
    return (u32x2){__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}
__device__ inline bool finite(float x) { return (f32_bits(x) & 0x7F800000u) != 0x7F800000u; }
// Whether a sum is NaN, or so large that four of them may pass fp32's range.
template <int N>
__device__ inline bool too_large(const f32x4 (&o)[N]) {
    float most = 0.0f;
    #pragma unroll
    for (int c = 0; c < N; ++c)
        #pragma unroll
        for (int j = 0; j < 4; ++j) most = __builtin_elementwise_maximum(most, __builtin_fabsf(o[c][j]));  // (NaN is more than all)
    return !(most < 0x1p125f);
}
// Four means, sums o times f, to bf16 or (a part) fp32; `second`: those that were not finite.
__device__ inline void put(__bf16* to, const f32x4& o, float f, bool second) {
    u32x2 x = bf16x4_of(o, f);
    if (second) {
        const u32x2 old = *reinterpret_cast<const u32x2*>(to);
        #pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t lost = (finite(bits_f32(old[i] << 16)) ? 0u : 0xFFFFu) | (finite(bits_f32(old[i])) ? 0u : 0xFFFF0000u);
            x[i] = (x[i] & lost) | (old[i] & ~lost);
        }
    }
    *reinterpret_cast<u32x2*>(to) = x;
}
__device__ inline void put(float* to, const f32x4& o, float f, bool second) {
    f32x4 x = o * f;
    if (second) {
        const f32x4 old = *reinterpret_cast<const f32x4*>(to);
        #pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = finite(old[i]) ? old[i] : x[i];
    }
    *reinterpret_cast<f32x4*>(to) = x;
}
// The upper halves of two values, their bf16 cut off; and those two as fp32.
__device__ inline uint32_t upper(float a, float b) { return __builtin_amdgcn_perm(f32_bits(b), f32_bits(a), 0x07060302u); }
__device__ inline float first_of(uint32_t two) { return bits_f32(two << 16); }
__device__ inline float second_of(uint32_t two) { return bits_f32(two & 0xFFFF0000u); }
// A barrier of the workgroup that waits for no load.
__device__ inline void meet_waves() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
// What scores are taken from, m as above (-inf: none yet; inf: NaN), or `lift` more.
__device__ inline float reference(float m, float lift = 0.0f) { return m == kNegInf ? 0.0f : m + (lift + (m - m)); }

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

// n / d rounded down, for quotients below 2^10 and d below 2^11 (by: the reciprocal of d, to the last place): (n + 1/2) / d is 2^-12
// at least from every whole number, of which three roundings of 2^-24 lose less.
__device__ inline uint32_t quotient(uint32_t n, float by) { return (uint32_t)(((float)n + 0.5f) * by); }

// n / d rounded down, for quotients below 2^22: the reciprocal leaves less than one.
__device__ inline uint32_t long_quotient(uint32_t n, uint32_t d) {
    const uint32_t q = (uint32_t)((float)n * __builtin_amdgcn_rcpf((float)d));
    return q * d > n ? q - 1 : n - q * d >= d ? q + 1 : q;
}

// What a wave's lane knows of sequence 64 chunk + lane.
struct Seq {
    int n, t0, T;      // rows held, first packed token, tokens
    int first, units;  // first unit, number of units (1 at least where T > 0)
    int tiles;         // of TILE query rows
    uint32_t segments; // tiles times KV heads
    uint32_t pair, head; // WIDE: units of two tiles, and of a KV head, with what beginnings count for
};

__device__ inline int clamp_token(const KvpAttendParams& p, int t) { return t < 0 ? 0 : t > p.tokens ? (int)p.tokens : t; }

template <int TILE>
__device__ inline Seq load_seq(const KvpAttendParams& p, int group, int s) {
    const KvpPages& g = p.pages;
    Seq q = {};
    if (s >= g.n_seq) return q;
    // (three loads on their way at once, whether there is a tok0 or not)
    const int32_t* tok0 = g.tok0 ? g.tok0 : g.lens;
    const int i = g.tok0 ? s : 0;
    q.n = g.lens[s];
    const int begin = tok0[i], end = tok0[g.tok0 ? i + 1 : 0];
    q.t0 = g.tok0 ? clamp_token(p, begin) : s;
    q.T = g.tok0 ? clamp_token(p, end) - q.t0 : s < p.tokens;
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
    q.tiles = (q.T * group + TILE - 1) / TILE;  // (tokens * heads fits 31 bits)
    q.segments = (uint32_t)q.tiles * (uint32_t)g.kv_heads;
    return q;
}

// The units that a tile of TILE rows sees, from the sequence's rows.
struct Units {
    int first, number;  // 1 at least
};
template <int TILE>
__device__ inline Units units_of_tile(const KvpAttendParams& p, int n, int T, int group, int tile) {
    const int last = (tile + 1) * TILE < T * group ? (tile + 1) * TILE : T * group;
    const int pos0 = n - T + divide(tile * TILE, p.by_group), end = n - T + divide(last - 1, p.by_group) + 1;
    const int lo = p.window > 0 && pos0 >= p.window ? pos0 - p.window + 1 : 0, hi = end < p.pages.capacity ? end : p.pages.capacity;
    const int first = lo / kKvpUnit, number = (hi + kKvpUnit - 1) / kKvpUnit - first;
    return {first, number < 1 ? 1 : number};
}
// What a KV head's tiles of TILE rows count for where runs are dealt out.  Later tiles see more: the first and the last of
// all (of an odd number: of all but the last), the second and the last but one, .. are pairs, of which none has more
// units than `pair`: tiles j and k, j + k = c, see 2 (n - T) + (TILE (c + 2) - 2) / group rows at most in all; with a window each sees
// that and what its own rows are apart.  (2048 tokens, 16 heads on 4 of 64, 128 and 256 channels, every tile counted as the last, first and last in
// turn: 69, 96 and 154 us; so 57, 70 and 111, when other parts took longer than now.)
template <int TILE>
__device__ inline void add_weights(const KvpAttendParams& p, Seq& q) {
    const int pairs = q.tiles / 2, capacity = p.pages.capacity;
    int one = q.units;
    if (p.window > 0) {
        const int most = (p.window < capacity ? p.window : capacity) + divide(TILE, p.by_group) + 3 * kKvpUnit;
        one = most / kKvpUnit < one ? most / kKvpUnit : one;
    }
    int pair = 2 * one;
    if (q.n >= q.T) {
        const int before = q.n - q.T < capacity ? q.n - q.T : capacity;
        const int both = (2 * before + divide(TILE * (2 * pairs + 1) - 2, p.by_group)) / kKvpUnit + 2;
        pair = both < pair ? both : pair;
    }
    q.pair = (uint32_t)(pair + 2 * p.begin);
    q.head = (uint32_t)pairs * q.pair + (q.tiles & 1 ? (uint32_t)(one + p.begin) : 0);
}

// Waves of a workgroup, and of a SIMD: as many as LDS and registers allow.
constexpr int waves_of(int nt, bool wide) { return wide && nt == 1 ? 8 : 4; }
constexpr int simd_waves(int d, int nt, bool wide) { return wide && nt == 1 ? 2 : d == 64 && nt == 2 ? 3 : 256 / d; }

// Tiles of 16 NT query rows, whose units the four waves take in turn, each by itself; or (WIDE) of 128, of which
// each wave has its share, and all of them every unit: a ring of four in LDS, which they fill together.
template <int D, int NT, bool WIDE>
__global__ __launch_bounds__(64 * waves_of(NT, WIDE), simd_waves(D, NT, WIDE)) void attend_kernel(const KvpAttendParams p) {
    constexpr int WAVES = waves_of(NT, WIDE), kTile = WIDE ? 16 * NT * WAVES : 16 * NT;
    constexpr int NJ = D / 32;                        // K: fragments of 32 channels
    constexpr int NC = D / 16;                        // V: blocks of 16 channels
    constexpr int kParts = WIDE ? 2 : 3;              // bf16 parts of a weight
    constexpr int kPitch = D + 4;
    constexpr int kSlot = kKvpUnit * D * 2;           // a unit of K, or of V
    __shared__ __attribute__((aligned(1024))) char lds[8 * kSlot];
    static_assert(8 * kSlot >= 4 * 16 * kPitch * 4, "o_s");
    __shared__ float ml_s[4][16][2], all_s[16][2];
    __shared__ __attribute__((aligned(16))) uint32_t lost_s[2][WAVES];  // (WIDE) waves with sums that are too large, of this segment and the next
    float (*o_s)[16][kPitch] = reinterpret_cast<float (*)[16][kPitch]>(lds);  // once the waves are through with K and V

    const KvpPages& g = p.pages;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int G = divide(p.heads, p.by_kv_heads);

    // the run [begin, end) of this workgroup
    const int chunks = (g.n_seq + 63) / 64;
    auto load = [&](int s) {
        Seq q = load_seq<kTile>(p, G, s);
        if (WIDE && q.T > 0) add_weights<kTile>(p, q);
        return q;
    };
    const uint32_t extra = (uint32_t)p.begin;
    auto run_of = [&](const Seq& q) -> uint32_t { return q.head * (uint32_t)g.kv_heads; };  // (WIDE)
    Seq q = load((int)(threadIdx.x & 63));
    uint32_t segments = scan_lanes(q.segments), units_to = scan_lanes(q.segments * (uint32_t)q.units), before = 0;
    uint32_t all_segments = lane_u32(segments, 63), all_units = lane_u32(units_to, 63);
    uint32_t run_to = WIDE ? scan_lanes(run_of(q)) : 0, all_runs = WIDE ? lane_u32(run_to, 63) : 0;
    for (int c = 1; c < chunks; ++c) {
        const Seq r = load(64 * c + (int)(threadIdx.x & 63));
        all_segments += lane_u32(scan_lanes(r.segments), 63);
        all_units += lane_u32(scan_lanes(r.segments * (uint32_t)r.units), 63);
        if (WIDE) all_runs += lane_u32(scan_lanes(run_of(r)), 63);
    }
    // Little work: segments are cut into even parts of `cut` units at most, a workgroup each (segments + units /
    // cut are no more than there are workgroups).  More: units in a row, each segment's with `extra` before them
    // for what its beginning costs, are dealt out in equal runs.
    uint32_t cut = 0;
    float by_cut = 0.0f;
    if (!p.whole && all_segments < p.wgs && all_units < (kMostCut + 1) * p.wgs) {
        cut = quotient(all_units, __builtin_amdgcn_rcpf((float)(p.wgs - all_segments))) + 1;
        if (cut < kLeastCut) cut = kLeastCut;
        if (cut > kMostCut) cut = 0;
        else by_cut = __builtin_amdgcn_rcpf((float)cut);
    }
    auto size_of = [&](uint32_t units) -> uint32_t { return cut ? quotient(units + cut - 1, by_cut) : units + extra; };
    const uint32_t total = cut ? p.wgs : WIDE ? all_runs : all_units + extra * all_segments, per = cut ? 1 : (total + p.wgs - 1) / p.wgs;
    auto weight_of = [&](const Seq& q) -> uint32_t { return WIDE && !cut ? run_of(q) : q.segments * size_of((uint32_t)q.units); };
    uint32_t scan = cut ? scan_lanes(weight_of(q)) : WIDE ? run_to : units_to + extra * segments;
    uint32_t w = blockIdx.x;
    // (runs behind each other to one XCD, w % 8 of the launch, whose L2 has what they share: 8192 tokens, 32 heads on 4 of 256 channels
    // fetch 0.4 GB and not 6.9; 16384 of 128 channels 4314 -> 4176 us)
    if (WIDE && !cut && !p.whole && p.wgs % 8 == 0) {
        const uint32_t some = ((total + per - 1) / per + 7) / 8;
        if (w / 8 >= some) return;
        w = w % 8 * some + w / 8;
    }
    const uint32_t begin = w * per;
    if (begin >= total) return;
    const uint32_t end = begin + per < total ? begin + per : total;

    const int rowb = g.kv_heads * D * 2;
    uint32_t at = begin;  // where in the run we are
    int chunk = 0;
    int turn = 0;         // of lost_s
    bool again = false;   // the waves have joined their sums in LDS
    bool second = false;  // the segment is taken again, for means that were not finite
    while (at < end) {
        const uint32_t start = at;
        const int tid = hidden((int)threadIdx.x), lane = tid & 63, li = lane & 15, grp = lane >> 4;
        // the sequence that `at` is in (tok0 that does not ascend may make this fail: the run ends)
        while (at - before >= lane_u32(scan, 63)) {
            before += lane_u32(scan, 63);
            if (++chunk >= chunks) return;
            q = load(64 * chunk + lane);
            scan = scan_lanes(weight_of(q));
        }
        const int s = __builtin_popcountll(__ballot(scan <= at - before));
        if (s > 63) return;
        const int n = lane_int(q.n, s), seq_t0 = lane_int(q.t0, s), T = lane_int(q.T, s);
        int units = lane_int(q.units, s), first_unit = lane_int(q.first, s);
        const uint32_t weight = lane_u32(weight_of(q), s), base = before + lane_u32(scan, s) - weight;
        if (at - base >= weight) return;
        // The segment that `at` is in, from seg0 to next: heads of a tile behind each other, as their rows lie in memory; or (WIDE,
        // unless cut) pairs of tiles of a head, and the last of an odd number.
        int segment, tile, h;
        uint32_t seg0, next;
        float by_size;
        if (WIDE && !cut) {
            const int tiles = lane_int(q.tiles, s), pairs = tiles / 2;
            const uint32_t pair = lane_u32(q.pair, s), head = lane_u32(q.head, s);
            h = (int)long_quotient(at - base, head);
            seg0 = base + (uint32_t)h * head;
            tile = (int)long_quotient(at - seg0, pair);
            const bool alone = tile >= pairs;
            if (alone) tile = pairs;
            seg0 += (uint32_t)tile * pair;
            next = alone ? base + (uint32_t)(h + 1) * head : seg0 + pair;
            if (alone) tile = tiles - 1;
            Units mine = units_of_tile<kTile>(p, n, T, G, tile);
            const uint32_t second = seg0 + (uint32_t)mine.number + extra;
            if (!alone && at >= second) {
                seg0 = second;
                tile = 2 * pairs - 1 - tile;
                mine = units_of_tile<kTile>(p, n, T, G, tile);
            } else if (!alone) {
                next = second;
            }
            units = mine.number;
            first_unit = mine.first;
        } else {
            const uint32_t size = size_of((uint32_t)units);
            by_size = __builtin_amdgcn_rcpf((float)size);
            segment = (int)(cut ? quotient(at - base, by_size) : (at - base) / size);
            seg0 = base + (uint32_t)segment * size;
            next = seg0 + size;
        }
        if (next <= at) return;  // (sums past 32 bits, of tok0 that does not ascend)
        const uint32_t unit0 = cut ? seg0 : seg0 + extra, unit1 = cut ? next : unit0 + (uint32_t)units;  // of its first unit, behind its last
        int u0 = 0, u1 = units;
        if (p.whole) {
            at = next;
            if (seg0 < begin) continue;  // its beginning was another workgroup's
        } else if (cut) {
            const int part = (int)quotient((uint32_t)units + (next - seg0) - 1, by_size);
            u0 = (int)(at - seg0) * part;
            u1 = u0 + part < units ? u0 + part : units;
            at = next;
        } else {
            u0 = at > unit0 ? (int)(at - unit0) : 0;
            u1 = end < unit1 ? (int)(end - unit0) : units;
            at = next;
            if (u1 <= 0 || (WIDE && u0 >= units)) continue;
        }
        if (g.pages == 0) u1 = u0;  // there is nothing to read
        if (!WIDE && again) __syncthreads();  // the other waves may still read the last segment's sums, which lie where K and V come
        again = true;
        const KvpAttendParams& args = *hidden_arguments<KvpAttendParams>();
        const KvpPages& gp = args.pages;
        if (!WIDE || cut) {
            tile = divide(segment, args.by_kv_heads);
            h = segment - tile * gp.kv_heads;
        }
        const float scale = args.scale_log2, unseen = scale < 0.0f ? -kNegInf : kNegInf;
        const float lift = second ? kAbove : 0.0f;
        const int seq = 64 * chunk + s;

        const int r0 = tile * kTile, rows = T * G - r0 < kTile ? T * G - r0 : kTile;
        // the wave's rows: row w0 + 16 i + li of the tile (those past the last repeat it); it sees the keys in (low, pos]
        const int w0 = WIDE ? wave * (16 * NT) : 0, my_rows = rows - w0 < 16 * NT ? rows - w0 : 16 * NT;
        auto my_row = [&](int i) { return r0 + (w0 + 16 * i + li < rows ? w0 + 16 * i + li : rows - 1); };
        int row_t[NT], pos[NT], low[NT];
        auto below = [&](int pos) { return args.window > 0 ? (pos < 0 ? -1 : pos - args.window) : -1; };
        #pragma unroll
        for (int i = 0; i < NT; ++i) {
            row_t[i] = divide(my_row(i), args.by_group);
            pos[i] = n - T + row_t[i];
            low[i] = below(pos[i]);
        }
        // positions of its first row and its last, and of the tile's
        auto pos_of = [&](int row) { return n - T + divide(r0 + (row < rows ? row : rows - 1), args.by_group); };
        const int pos0 = pos_of(w0), pos1 = pos_of(w0 + 16 * NT - 1), low0 = below(pos0), low1 = below(pos1);
        const int tile_pos1 = WIDE ? pos_of(kTile - 1) : pos1, tile_low0 = WIDE ? below(pos_of(0)) : low0;

        // Where a wave's next 64 units have their two groups of 16 rows in the pools, a lane each (a wave has every fourth
        // unit from u0 + wave on, or (WIDE) every one); -1: on no page.
        int64_t off[2];
        uint64_t todo = 0, whole = 0;  // bits of the units that some row of the tile sees, and of those that every row of the wave sees all of
        const int32_t* table = gp.table + (int64_t)seq * gp.table_stride;
        auto unit_of = [&](int step) { return WIDE ? u0 + step : u0 + wave + 4 * step; };
        auto look_up = [&](int step0) {
            const int u = unit_of(step0 + lane), r = (first_unit + u) * kKvpUnit;
            bool there[2];
            int page[2], rest[2];
            #pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int rt = r + 16 * t;
                there[t] = u < u1 && rt < gp.capacity && rt <= tile_pos1;
                const int column = there[t] ? divide(rt, gp.by_page) : 0;
                rest[t] = rt - column * gp.page;
                page[t] = table[column];
            }
            #pragma unroll
            for (int t = 0; t < 2; ++t) {
                there[t] = there[t] && (uint32_t)page[t] < (uint32_t)gp.pages;
                off[t] = there[t] ? (int64_t)page[t] * gp.page_stride + (int64_t)rest[t] * rowb : -1;
            }
            todo = __ballot((there[0] || there[1]) && r + kKvpUnit - 1 > tile_low0);
            whole = __ballot(there[0] && there[1] && r + kKvpUnit - 1 <= pos0 && r > low1);
        };
        auto lane_i64 = [&](int64_t x, int i) -> int64_t {
            return (int64_t)((uint64_t)lane_u32((uint32_t)(x >> 32), i) << 32 | lane_u32((uint32_t)x, i));
        };

        // the query rows, before the table is asked
        bf16x8 qf[NT][NJ];
        #pragma unroll
        for (int i = 0; i < NT; ++i) {
            const int row = my_row(i);
            const global_bytes src = (global_bytes)args.q.p + (int64_t)(seq_t0 + row_t[i]) * args.q.token +
                                     (int64_t)(h * G + (row - row_t[i] * G)) * args.q.head + 16 * grp;
            #pragma unroll
            for (int j = 0; j < NJ; ++j) qf[i][j] = *(const bf16x8 __attribute__((address_space(1)))*)(src + 64 * j);
        }

        f32x4 acc[NT][NC];  // channels 16 c + 4 grp ..
        float m[NT], from[NT], l[NT];  // from: reference(m, lift)
        #pragma unroll
        for (int i = 0; i < NT; ++i) {
            m[i] = kNegInf;
            from[i] = 0.0f;
            l[i] = 0.0f;
            #pragma unroll
            for (int c = 0; c < NC; ++c) acc[i][c] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
        }

        // Units in LDS, a slot for K and one for V behind it to each wave (WIDE: to each place of the ring): rows of D channels, in
        // which 16 bytes (K: those of channels 8 c .. at the place of c ^ fold_k(row)) or 32 (V: 16 c .., c ^ fold_v(row)) change
        // places, so that reads of 16 rows meet all banks.  An instruction brings 1 KiB: kRows rows, a lane 16 bytes.
        constexpr int kRows = 512 / D, kLoads = kKvpUnit / kRows;
        const int lane_row = lane / (D / 8), piece = lane % (D / 8);
        const uint32_t lane_at = (uint32_t)(lane_row * rowb + h * D * 2);
        const uint32_t kvoff = lane_at + ((piece ^ fold_k<D>(lane_row)) << 4);
        const uint32_t vvoff = lane_at + (((piece >> 1) ^ fold_v<D>(lane_row)) << 5) + ((piece & 1) << 4);
        const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_bytes)lds;  // (a multiple of the slots, which exchanges leave alone)
        int place = WIDE ? 0 : wave;
        const uint32_t kread = lds_at + (uint32_t)(li * D * 2 + ((grp ^ fold_k<D>(li)) << 4));
        const int vrow = 4 * grp + (li >> 2);
        const uint32_t vread = lds_at + (uint32_t)(kSlot + vrow * D * 2 + (fold_v<D>(vrow) << 5) + 8 * (li & 3));
        const global_bytes kb = (global_bytes)gp.k, vb = (global_bytes)gp.v;
        // (folds are linear: that of lane_row + row is fold(lane_row) ^ fold(row))
        auto load_k = [&](const int64_t (&a)[2]) {
            const uint32_t from = hidden(kvoff);
            const lds_bytes to = (lds_bytes)lds + place * (2 * kSlot);
            #pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int row = i * kRows % 16;
                load_lds<true>(kb + a[i * kRows / 16] + row * rowb + (from ^ (uint32_t)(fold_k<D>(row) << 4)), to + i * 1024);
            }
        };
        auto load_v = [&](const int64_t (&a)[2]) {
            const uint32_t from = hidden(vvoff);
            const lds_bytes to = (lds_bytes)lds + place * (2 * kSlot) + kSlot;
            #pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int row = i * kRows % 16;
                load_lds<true>(vb + a[i * kRows / 16] + row * rowb + (from ^ (uint32_t)(fold_v<D>(row) << 5)), to + i * 1024);
            }
        };
        // A wave's share of a unit of K and V, to a place of the ring.
        constexpr int kShare = kLoads / WAVES;
        auto load_share = [&](const int64_t (&a)[2], int to) {
            const uint32_t k_from = hidden(kvoff), v_from = hidden(vvoff);
            const int64_t at = a[wave * 2 / WAVES];
            #pragma unroll
            for (int i = 0; i < kShare; ++i) {
                const int row = (wave * kShare + i) * kRows % 16;
                const lds_bytes slot = (lds_bytes)lds + to * (2 * kSlot) + (wave * kShare + i) * 1024;
                load_lds<!WIDE>(kb + at + row * rowb + (k_from ^ (uint32_t)(fold_k<D>(row) << 4)), slot);
                load_lds<!WIDE>(vb + at + row * rowb + (v_from ^ (uint32_t)(fold_v<D>(row) << 5)), slot + kSlot);
            }
        };
        float x[NT][8];
        auto scores = [&]() {
            const uint32_t from = hidden(kread) + (uint32_t)(place * (2 * kSlot));
            f32x4 sums[NT][2];
            #pragma unroll
            for (int i = 0; i < NT; ++i) sums[i][0] = sums[i][1] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
            constexpr int kAtOnce = NT > 1 && NJ > 4 ? 2 : NJ;
            #pragma unroll
            for (int j0 = 0; j0 < NJ; j0 += kAtOnce) {
                uint32_t at[kAtOnce];
                u32x4 k[2 * kAtOnce];
                #pragma unroll
                for (int j = 0; j < kAtOnce; ++j) at[j] = from ^ (uint32_t)((j0 + j) << 6);
                if constexpr (kAtOnce == 2) read_k2<16 * D * 2>(at, k);
                else if constexpr (kAtOnce == 4) read_k4<16 * D * 2>(at, k);
                else read_k8<16 * D * 2>(at, k);
                #pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    #pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        sums[i][0] = dev::mma(__builtin_bit_cast(bf16x8, k[2 * j]), qf[i][j0 + j], sums[i][0]);
                        sums[i][1] = dev::mma(__builtin_bit_cast(bf16x8, k[2 * j + 1]), qf[i][j0 + j], sums[i][1]);
                    }
            }
            #pragma unroll
            for (int i = 0; i < NT; ++i)
                #pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] = sums[i][e / 4][e % 4];
        };
        // x, products not yet scaled, becomes the weights.  Their parts are cut off, not rounded, and what is left has 2^-24 of the first (2^-16 of the
        // second, 2^-20 where there are two) added, so that it is above zero, and an infinity in V, times all parts, is one.
        auto weigh = [&](bf16x8 (&w)[kParts][NT]) {
            float top[NT];
            bool above = false;
            if (scale < 0.0f) {
                #pragma unroll
                for (int i = 0; i < NT; ++i) {
                    top[i] = x[i][0];
                    #pragma unroll
                    for (int e = 1; e < 8; ++e) top[i] = __builtin_fminf(top[i], x[i][e]);
                    top[i] = -top[i];
                }
            } else {
                #pragma unroll
                for (int i = 0; i < NT; ++i) {
                    top[i] = x[i][0];
                    #pragma unroll
                    for (int e = 1; e < 8; ++e) top[i] = __builtin_fmaxf(top[i], x[i][e]);
                }
            }
            #pragma unroll
            for (int i = 0; i < NT; ++i) {
                top[i] = group_max(top[i]) * __builtin_fabsf(scale);
                above |= top[i] > m[i] + kBehind;
            }
            if (__any(above)) {
                #pragma unroll
                for (int i = 0; i < NT; ++i) {
                    top[i] = top[i] > m[i] + kBehind ? top[i] : m[i];
                    const float fade = m[i] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(from[i] - reference(top[i], lift));
                    m[i] = top[i];
                    from[i] = reference(top[i], lift);
                    l[i] *= fade;
                    #pragma unroll
                    for (int c = 0; c < NC; ++c) acc[i][c] *= fade;
                }
            }
            #pragma unroll
            for (int i = 0; i < NT; ++i) {
                float sum = 0.0f;
                #pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[i][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i][e], scale, -from[i]));
                    sum += x[i][e];
                }
                l[i] += sum;
                u32x4 part[kParts];
                #pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    // (what is left of the two values)
                    float r0 = x[i][e], r1 = x[i][e + 1];
                    #pragma unroll
                    for (int k = 0; k + 1 < kParts; ++k) {
                        const float less = (kParts == 2 ? 0x1p-20f : k == 0 ? 0x1p-24f : 0x1p-16f) - 1.0f;
                        part[k][e / 2] = upper(r0, r1);
                        r0 = __builtin_fmaf(first_of(part[k][e / 2]), less, r0);
                        r1 = __builtin_fmaf(second_of(part[k][e / 2]), less, r1);
                    }
                    part[kParts - 1][e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){r0, r1}, bf16x2));
                }
                #pragma unroll
                for (int k = 0; k < kParts; ++k) w[k][i] = __builtin_bit_cast(bf16x8, part[k]);
            }
        };
        // In a unit that some row does not see in full, or that lies on no page in part (there: the halves that are on
        // one), a key that a row does not see has to leave the product, as its V may hold an infinity or NaN, of which
        // no weight makes zero.  Keys that no row sees are cleared, and where rows see different ones, such
        // values of all keys are; they are put back, row by row, from memory (at: the unit's).
        auto seen = [&](int r, int there, int e, int first, int last) {  // key e lies on a page and in (first, last]
            const int key = r + 4 * grp + (e < 4 ? e : 12 + e);
            return (there >> (e / 4) & 1) && key <= last && key > first;
        };
        // (all: every row sees all of the unit.  Products of their own for it had the compiler keep the sums in two places: 32 to 45
        // registers more, and 16384 tokens of 128 and 256 channels 3.89 and 8.33 ms, so 3.72 and 8.01.)
        auto add_values = [&](bool all, int r, int there, const int64_t (&at)[2], const bf16x8 (&w)[kParts][NT]) {
            uint32_t keep[4] = {};  // bits of keys 2i and 2i + 1
            if (!all) {
                #pragma unroll
                for (int i = 0; i < 4; ++i)
                    keep[i] = (seen(r, there, 2 * i, low0, pos1) ? 0xFFFFu : 0u) | (seen(r, there, 2 * i + 1, low0, pos1) ? 0xFFFF0000u : 0u);
            }
            const bool mixed = pos0 != pos1;
            bool found = false;
            const uint32_t from_v = hidden(vread) + (uint32_t)(place * (2 * kSlot));
            constexpr int kAtOnce = NC < 8 || NT > 1 ? 4 : 8;
            #pragma unroll
            for (int c0 = 0; c0 < NC; c0 += kAtOnce) {
                uint32_t from[kAtOnce];
                u32x2 pair[2 * kAtOnce];
                u32x4 v[kAtOnce];  // the eight keys of a lane in channel 16 c + li
                #pragma unroll
                for (int c = 0; c < kAtOnce; ++c) from[c] = from_v ^ (uint32_t)((c0 + c) << 5);
                if constexpr (kAtOnce == 4) read_v4<16 * D * 2>(from, pair);
                else read_v8<16 * D * 2>(from, pair);
                #pragma unroll
                for (int c = 0; c < kAtOnce; ++c) v[c] = (u32x4){pair[2 * c][0], pair[2 * c][1], pair[2 * c + 1][0], pair[2 * c + 1][1]};
                if (!all) {
                    #pragma unroll
                    for (int c = 0; c < kAtOnce; ++c)
                        #pragma unroll
                        for (int i = 0; i < 4; ++i) v[c][i] &= keep[i];
                    if (mixed) {
                        #pragma unroll
                        for (int c = 0; c < kAtOnce; ++c)
                            #pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t out = ((v[c][i] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((v[c][i] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
                                found |= out != 0;
                                v[c][i] &= ~out;
                            }
                    }
                }
                #pragma unroll
                for (int c = 0; c < kAtOnce; ++c)
                    #pragma unroll
                    for (int i = 0; i < NT; ++i)
                        #pragma unroll
                        for (int k = 0; k < kParts; ++k) acc[i][c0 + c] = dev::mma(__builtin_bit_cast(bf16x8, v[c]), w[k][i], acc[i][c0 + c]);
            }
            if (!__any(found)) return;
            #pragma unroll 1
            for (int t = 0; t < kKvpUnit; ++t) {
                const int key = r + t, e = (t & 3) + (t >= 16 ? 4 : 0);
                if (!(there >> (t / 16) & 1) || key > pos1 || key <= low0) continue;  // (uniform)
                const global_bytes from = vb + at[t / 16] + (int64_t)(t % 16) * rowb + (uint32_t)(h * D * 2 + 8 * grp);
                float weight[NT];
                #pragma unroll
                for (int i = 0; i < NT; ++i) {
                    float mine = x[i][0];
                    #pragma unroll
                    for (int k = 1; k < 8; ++k) mine = e == k ? x[i][k] : mine;
                    weight[i] = __shfl(mine, li + 16 * (t % 16 / 4));
                }
                #pragma unroll
                for (int c = 0; c < NC; ++c) {
                    __builtin_amdgcn_sched_barrier(0);
                    const u32x2 four = *(const u32x2 __attribute__((address_space(1)))*)(from + 32 * c);
                    #pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float value = bits_f32(j & 1 ? four[j / 2] & 0xFFFF0000u : four[j / 2] << 16);
                        const bool back = (f32_bits(value) & 0x7F800000u) == 0x7F800000u;
                        #pragma unroll
                        for (int i = 0; i < NT; ++i)
                            if (back && key <= pos[i] && key > low[i]) acc[i][c][j] += weight[i] * value;
                    }
                }
            }
        };

        // (of a half on no page, rows of the first one are read, and count for nothing)
        int64_t a[2];
        int there;
        auto where = [&](int j) {
            a[0] = lane_i64(off[0], j);
            a[1] = lane_i64(off[1], j);
            there = 0;
            #pragma unroll
            for (int t = 0; t < 2; ++t) {
                if ((int)(a[t] >> 32) >= 0) there |= 1 << t;
                else a[t] = 0;
            }
        };
        auto hide_unseen = [&](int r, int there) {
            #pragma unroll
            for (int i = 0; i < NT; ++i)
                #pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] = seen(r, there, e, low[i], pos[i]) ? x[i][e] : unseen;
        };
        const int steps = WIDE ? u1 - u0 : u1 - u0 > wave ? (u1 - u0 - wave + 3) / 4 : 0;
        for (int step0 = 0; step0 < steps; step0 += 64) {
            look_up(step0);
            if (todo == 0) continue;
            if constexpr (WIDE) {
                // Three units are on their way while one is in work.  A barrier for each: what the waves have loaded of it is
                // there, and its predecessor's place is free.
                uint64_t ahead = todo;
                int to = 0;
                auto load_next = [&]() {
                    where(__builtin_ctzll(ahead));
                    ahead &= ahead - 1;
                    load_share(a, to);
                    to = (to + 1) & 3;
                };
                meet_waves();  // the last 64 units' places are free
                #pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (ahead) load_next();
                place = 0;
                while (todo) {
                    const int j = __builtin_ctzll(todo), left = __builtin_popcountll(todo);
                    todo &= todo - 1;
                    if (left > 2) wait_loads<4 * kShare>();
                    else if (left > 1) wait_loads<2 * kShare>();
                    else wait_loads<0>();
                    meet_waves();
                    if (ahead) load_next();
                    const int r = (first_unit + unit_of(step0 + j)) * kKvpUnit;
                    if (my_rows > 0 && r <= pos1 && r + kKvpUnit - 1 > low0) {
                        const bool all = whole >> j & 1;
                        where(j);
                        scores();
                        if (!all) hide_unseen(r, there);
                        bf16x8 w[kParts][NT];
                        weigh(w);
                        add_values(all, r, there, a, w);
                    }
                    place = (place + 1) & 3;
                }
                continue;
            }
            int j = __builtin_ctzll(todo);
            where(j);
            wait_lds();  // the last reads of both slots
            load_k(a);
            load_v(a);
            for (;;) {
                // The next K is on its way once its slot has been read, the next V likewise: loads come in order, so
                // those behind the ones that are waited for tell how many may be outstanding.
                todo &= todo - 1;
                const bool more = todo != 0;
                const int r = (first_unit + unit_of(step0 + j)) * kKvpUnit, there_now = there;
                const int64_t now[2] = {a[0], a[1]};
                const bool all = whole >> j & 1;
                wait_loads<kLoads>();  // K: V's are behind it
                scores();
                if (more) {
                    j = __builtin_ctzll(todo);
                    where(j);
                    wait_lds();
                    load_k(a);
                }
                if (!all) hide_unseen(r, there_now);
                bf16x8 w[kParts][NT];
                weigh(w);
                if (more) wait_loads<kLoads>();  // V: the next K's are behind it
                else wait_loads<0>();
                add_values(all, r, there_now, now, w);
                if (!more) break;
                wait_lds();
                load_v(a);
            }
        }

        const KvpAttendParams& late = *hidden_arguments<KvpAttendParams>();
        // whether the segment's first unit is of this run, and all of them
        const bool begins = late.whole || unit0 >= begin, one = late.whole || (begins && unit1 <= end);
        const int64_t part0 = (int64_t)(2 * w + (begins ? 1 : 0)) * kTile;
        auto out_row = [&](int rr) -> int64_t {
            const int t = divide(r0 + rr, late.by_group);
            return (int64_t)(seq_t0 + t) * late.heads + h * G + (r0 + rr - t * G);
        };
        auto row_done = [&](int rr, float m, float l) {
            const int64_t to = out_row(rr);
            if (!one) *reinterpret_cast<f32x2*>(late.part_ml + (part0 + rr) * 2) = (f32x2){m, l};
            else if (late.lse) late.lse[to] = (reference(m) + __builtin_amdgcn_logf(l)) * kLn2;
            if (!late.whole && begins) late.meta[to] = (uint64_t)rr << 48 | (uint64_t)((unit1 - 1) / per - w + 1) << 24 | w;
        };
        bool lost = false;
        if constexpr (WIDE) {  // a row's values from the lanes that have them
            #pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int rr = w0 + 16 * i + li;
                const float my_l = group_sum(l[i]);
                if (rr >= rows) continue;
                lost |= too_large(acc[i]);
                const float inv = my_l > 0.0f || my_l != my_l ? 1.0f / my_l : 0.0f;
                float* part = late.part_o + (part0 + rr) * D + 4 * grp;
                __bf16* out = static_cast<__bf16*>(late.o) + out_row(rr) * D + 4 * grp;
                #pragma unroll
                for (int c = 0; c < NC; ++c) {
                    if (one) put(out + 16 * c, acc[i][c], inv, second);
                    else put(part + 16 * c, acc[i][c], inv, second);
                }
                if (grp == 0 && !second) row_done(rr, m[i], my_l);
            }
            const bool any = __any(lost);
            if (lane == 0) lost_s[turn][wave] = any;
            wait_lds();
            meet_waves();
            u32x4 x[2] = {};
            read_words<WAVES>((uint32_t)(uintptr_t)(lds_bytes)&lost_s[turn][0], x);
            const uint32_t all = x[0][0] | x[0][1] | x[0][2] | x[0][3] | x[1][0] | x[1][1] | x[1][2] | x[1][3];
            turn ^= 1;
            second = !second && __builtin_amdgcn_readfirstlane((int)all);
            if (second) at = start;
            continue;
        }
        #pragma unroll
        for (int i = 0; i < NT; ++i) {
            if (16 * i >= rows) break;
            const float my_l = group_sum(l[i]);
            __syncthreads();  // K and V, and the values before these, are done with
            const uint32_t sign = __any(too_large(acc[i])) ? 0x80000000u : 0u;  // goes with the sums of weights, which have none
            if (grp == 0) {
                ml_s[wave][li][0] = m[i];
                ml_s[wave][li][1] = bits_f32(f32_bits(my_l) | sign);
            }
            __syncthreads();
            float top = kNegInf, sum = 0.0f;
            #pragma unroll
            for (int k = 0; k < 4; ++k) top = __builtin_fmaxf(top, ml_s[k][li][0]);
            const float from = reference(top);
            #pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float weights = __builtin_fabsf(ml_s[k][li][1]);
                lost |= (int)f32_bits(ml_s[k][li][1]) < 0;
                sum += ml_s[k][li][0] == kNegInf ? weights : weights * __builtin_amdgcn_exp2f(reference(ml_s[k][li][0]) - from);
            }
            const float fade = m[i] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(reference(m[i]) - from);
            // (m is -inf where the wave saw nothing: zeros; or only NaN, which stays)
            #pragma unroll
            for (int c = 0; c < NC; ++c) *reinterpret_cast<f32x4*>(&o_s[wave][li][16 * c + 4 * grp]) = acc[i][c] * fade;
            if (tid < 16) {  // wave 0: lane = row
                all_s[li][0] = top;
                all_s[li][1] = sum;
            }
            __syncthreads();
            constexpr int kPer = D / 4;  // threads of a row
            #pragma unroll
            for (int k = 0; k < 16 * kPer / kThreads; ++k) {
                const int r16 = (k * kThreads + hidden(tid)) / kPer, rr = 16 * i + r16, c = (tid % kPer) * 4;
                if (rr >= rows) continue;
                f32x4 o = *reinterpret_cast<const f32x4*>(&o_s[0][r16][c]);
                #pragma unroll
                for (int j = 1; j < 4; ++j) o += *reinterpret_cast<const f32x4*>(&o_s[j][r16][c]);
                const float z = all_s[r16][1], inv = z > 0.0f || z != z ? 1.0f / z : 0.0f;
                if (one) put(static_cast<__bf16*>(late.o) + out_row(rr) * D + c, o, inv, second);
                else put(late.part_o + (part0 + rr) * D + c, o, inv, second);
            }
            if (!second && tid < 16 && 16 * i + tid < rows) row_done(16 * i + tid, all_s[tid][0], all_s[tid][1]);
        }
        second = !second && __any(lost);  // (the same in every wave)
        if (second) at = start;
    }
}

// Parts put together: m as above, l the sum of weights, o the mean of the values, which stays in the range of the parts' means.
struct Joined {
    float m = kNegInf, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    template <int N>
    __device__ inline void add(const f32x2 (&ml)[N], const f32x4 (&mean)[N]) {
        float top = m, e[N];
        #pragma unroll
        for (int k = 0; k < N; ++k) top = __builtin_fmaxf(top, ml[k][0]);
        const float from = reference(top), f = l * (m == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(reference(m) - from));
        l = f;
        #pragma unroll
        for (int k = 0; k < N; ++k) {
            e[k] = ml[k][1] * (ml[k][0] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(reference(ml[k][0]) - from));
            l += e[k];
        }
        const float by = l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(l);
        o *= f * by;
        #pragma unroll
        for (int k = 0; k < N; ++k) o += mean[k] * (e[k] * by);
        m = top;
    }
};

// Parts `begin`, begin + step, .. of a row that begins in workgroup w's slots, the four channels from c on, with the loads
// of four parts on their way.
template <int D>
__device__ inline Joined join_parts(const KvpAttendParams& p, uint32_t w, uint32_t parts, int row, uint32_t begin, uint32_t step, int c) {
    constexpr int kAhead = 4;
    Joined sum;
    for (uint32_t i0 = begin; i0 < parts; i0 += kAhead * step) {
        f32x2 a[kAhead];
        f32x4 x[kAhead];
        #pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint32_t i = i0 + k * step < parts ? i0 + k * step : i0;
            const int64_t slot = 2 * (int64_t)(w + i) + (i == 0 ? 1 : 0);
            a[k] = *(const f32x2 __attribute__((address_space(1)))*)(p.part_ml + (slot * p.tile + row) * 2);
            x[k] = *(const f32x4 __attribute__((address_space(1)))*)(p.part_o + (slot * p.tile + row) * D + c);
        }
        #pragma unroll
        for (int k = 1; k < kAhead; ++k)
            if (i0 + k * step >= parts) {  // there is none
                a[k] = (f32x2){kNegInf, 0.0f};
                x[k] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
            }
        sum.add(a, x);
    }
    return sum;
}

// Joins the parts of rows.  With FEW rows a workgroup has 64 channels of one, and 16 threads to a part, so that many parts
// are read at once; else it has four rows, a wave each where they have few parts, and all of it one after another where
// they have more.
template <int D, bool FEW>
__global__ __launch_bounds__(kThreads) void join_kernel(const KvpAttendParams p) {
    constexpr int kPer = FEW ? 16 : D / 4, kWays = kThreads / kPer, kBlocks = FEW ? D / 64 : 1, kRows = FEW ? 1 : 4;
    constexpr int kWave = 64 / (D / 4);  // parts that a wave reads side by side
    __shared__ __attribute__((aligned(16))) float o_s[kWays][4 * kPer];
    __shared__ float m_s[kWays], l_s[kWays];
    const KvpPages& g = p.pages;
    const int64_t block = (int64_t)blockIdx.y * kFp8GridX + blockIdx.x, first = block / kBlocks * kRows, all = p.tokens * p.heads;
    if (first >= all) return;
    const int tid = (int)threadIdx.x, channel0 = (int)(block % kBlocks) * 64;
    // rows that no sequence has: nothing was written for them
    const int32_t* tok0 = g.tok0 ? g.tok0 : g.lens;
    const int begin = tok0[0], end = tok0[g.tok0 ? g.n_seq : 0];
    const int64_t low = (int64_t)(g.tok0 ? clamp_token(p, begin) : 0) * p.heads, high = (int64_t)(g.tok0 ? clamp_token(p, end) : g.n_seq) * p.heads;
    uint64_t meta[kRows];
    #pragma unroll
    for (int i = 0; i < kRows; ++i) meta[i] = p.meta[first + i < all ? first + i : first];
    auto parts_of = [&](int i) -> uint32_t {
        const uint32_t parts = (uint32_t)(meta[i] >> 24) & 0xFFFFFFu, w = (uint32_t)meta[i] & 0xFFFFFFu;
        return first + i >= low && first + i < high && first + i < all && w < p.wgs && parts <= p.wgs - w && parts >= 2 ? parts : 0;
    };
    auto write = [&](int64_t row, const Joined& x, int c) {
        *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.o) + row * D + c) = bf16x4_of(x.o, 1.0f);
        if (c == 0 && p.lse) p.lse[row] = (reference(x.m) + __builtin_amdgcn_logf(x.l)) * kLn2;
    };
    if constexpr (!FEW) {
        const int wave = tid / 64, lane = tid % 64, c = lane % (D / 4) * 4;
        uint64_t mine = meta[0];
        uint32_t parts = parts_of(0);
        #pragma unroll
        for (int i = 1; i < kRows; ++i) {
            if (wave == i) {
                mine = meta[i];
                parts = parts_of(i);
            }
        }
        if (parts > 0 && parts <= 4 * kWave) {
            Joined x = join_parts<D>(p, (uint32_t)mine & 0xFFFFFFu, parts, (int)(mine >> 48) & (p.tile - 1), (uint32_t)(lane / (D / 4)), kWave, c);
            #pragma unroll
            for (int step = D / 4; step < 64; step *= 2) {
                const f32x2 ml[1] = {(f32x2){__shfl_xor(x.m, step), __shfl_xor(x.l, step)}};
                f32x4 mean[1];
                #pragma unroll
                for (int j = 0; j < 4; ++j) mean[0][j] = __shfl_xor(x.o[j], step);
                x.add(ml, mean);
            }
            if (lane < D / 4) write(first + wave, x, c);
        }
    }
    #pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t parts = parts_of(i);
        if (parts == 0 || (!FEW && parts <= 4 * kWave)) continue;
        const int way = tid / kPer, c = tid % kPer * 4;
        Joined x = join_parts<D>(p, (uint32_t)meta[i] & 0xFFFFFFu, parts, (int)(meta[i] >> 48) & (p.tile - 1), (uint32_t)way, kWays, channel0 + c);
        __syncthreads();
        if (c == 0) m_s[way] = x.m;
        __syncthreads();
        float top = kNegInf;
        #pragma unroll
        for (int j = 0; j < kWays; ++j) top = __builtin_fmaxf(top, m_s[j]);
        const float weight = x.l * (x.m == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(reference(x.m) - reference(top)));
        *reinterpret_cast<f32x4*>(&o_s[way][c]) = x.o;
        if (c == 0) l_s[way] = weight;
        __syncthreads();
        if (way) continue;
        Joined y;
        y.m = top;
        #pragma unroll
        for (int j = 0; j < kWays; ++j) y.l += l_s[j];
        const float by = y.l == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(y.l);
        #pragma unroll
        for (int j = 0; j < kWays; ++j) y.o += *reinterpret_cast<const f32x4*>(&o_s[j][c]) * (l_s[j] * by);
        write(first + i, y, channel0 + c);
    }
}

// Workgroups of the join at most with 16 threads to a part: 192 tokens x 16 heads of 128 channels, two parts each, took 32.6 us
// so (the whole call) and 30.1 with four rows to a workgroup; 32 rows of 57 parts of 256 channels 21.2 and 31.7.
constexpr uint64_t kFewRows = 1024;

// Of 256 channels the sums of 16 rows to a wave leave registers for two waves on a SIMD.
template <int D>
constexpr int kWideTiles = D == 256 ? 1 : 2;

template <int D>
hipError_t launch(const KvpAttendParams& p, hipStream_t stream) {
    void* args[] = {const_cast<KvpAttendParams*>(&p)};
    const void* kernel = p.tile == 16 ? reinterpret_cast<const void*>(&attend_kernel<D, 1, false>)
                       : p.tile == 32 ? reinterpret_cast<const void*>(&attend_kernel<D, 2, false>)
                                      : reinterpret_cast<const void*>(&attend_kernel<D, kWideTiles<D>, true>);
    const uint32_t threads = p.tile == 128 ? 64 * (uint32_t)waves_of(kWideTiles<D>, true) : kThreads;
    const hipError_t e = hipLaunchKernel(kernel, dim3(p.wgs), dim3(threads), args, 0, stream);
    if (e != hipSuccess || p.whole) return e;
    const uint64_t rows = (uint64_t)p.tokens * (uint64_t)p.heads;
    if (rows * (D / 64) <= kFewRows)
        return hipLaunchKernel(reinterpret_cast<const void*>(&join_kernel<D, true>), wide_grid(rows * (D / 64)), dim3(kThreads), args, 0, stream);
    return hipLaunchKernel(reinterpret_cast<const void*>(&join_kernel<D, false>), wide_grid((rows + 3) / 4), dim3(kThreads), args, 0, stream);
}

}  // namespace

hipError_t launch_kvp_attend(const KvpAttendParams& p, hipStream_t stream) {
    return p.d == 64 ? launch<64>(p, stream) : p.d == 128 ? launch<128>(p, stream) : launch<256>(p, stream);
}

}  // namespace cap
