// Host side of the block-scaled FP8 KV cache: argument checks and launch plans
// of kvb_append, kvb_attend and kvb_select.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kvb.h"

namespace {

using cap::kKvbBlock;

struct Range { uint64_t a, b; };

uint64_t addr(const void* p) { return (uint64_t)(uintptr_t)p; }
Range range(const void* p, uint64_t bytes) { return {addr(p), addr(p) + (p ? bytes : 0)}; }
bool meet(const Range& x, const Range& y) { return x.a < y.b && y.a < x.b; }
bool wraps(const Range& x) { return x.b < x.a; }  // past the last address
uint64_t up(uint64_t x, uint64_t m) { return (x + m - 1) / m * m; }

// The sizes that every call shares.
int check_sizes(const kvb_seq* seqs, int32_t n_seq, int32_t heads, int32_t kv_heads, int32_t d, int32_t in_dtype,
                int64_t tokens) {
    if (n_seq < 0 || (n_seq > 0 && !seqs) || heads < 1 || kv_heads < 1 || d < 1) return CAP_E_INVAL;
    if (in_dtype != CAP_DTYPE_BF16 && in_dtype != CAP_DTYPE_F32) return CAP_E_INVAL;
    if (heads % kv_heads != 0) return CAP_E_INVAL;
    if (n_seq > KVB_MAX_SEQ || in_dtype != CAP_DTYPE_BF16 || (d != 64 && d != 128 && d != 256)) return CAP_E_UNSUPPORTED;
    // 32-bit offsets inside a block, and grids
    if ((int64_t)kKvbBlock * kv_heads * d > 0x7fffffff || (int64_t)heads * d > 0x7fffffff) return CAP_E_UNSUPPORTED;
    int64_t sum = 0;
    for (int32_t i = 0; i < n_seq; ++i) {
        const kvb_seq& s = seqs[i];
        if (s.rows < 0 || s.rows % kKvbBlock != 0 || s.n < 0 || s.T < 0 || s.T > s.n) return CAP_E_INVAL;
        if (s.rows > (int64_t)1 << 31) return CAP_E_UNSUPPORTED;
        if (s.n > s.rows) return CAP_E_SIZE;
        sum += s.T;
    }
    if (sum != tokens) return CAP_E_INVAL;
    return tokens > 0x7fffffff / heads ? CAP_E_UNSUPPORTED : CAP_OK;
}

// Elements between tokens of a packed tensor (0: contiguous) as bytes.
int check_stride(int64_t stride, int64_t width, int64_t* bytes) {
    if (stride == 0) stride = width;
    if (stride < width) return CAP_E_INVAL;
    if (stride > (int64_t)1 << 30) return CAP_E_UNSUPPORTED;
    if (stride % 8 != 0) return CAP_E_ALIGN;
    *bytes = stride * 2;
    return CAP_OK;
}

uint64_t span(int64_t tokens, int64_t stride_bytes, int64_t width) {
    return tokens == 0 ? 0 : (uint64_t)((tokens - 1) * stride_bytes + width * 2);
}

enum { K, V, SCALES, BOUNDS, OPEN, PARTS };

Range part(const kvb_seq& s, int which, int64_t row) {
    const int64_t nb = s.rows / kKvbBlock;
    switch (which) {
        case K: return range(s.k, (uint64_t)(s.rows * row));
        case V: return range(s.v, (uint64_t)(s.rows * row));
        case SCALES: return range(s.scales, (uint64_t)(nb * 8) * (uint64_t)row);  // row: kv_heads
        case BOUNDS: return range(s.bounds, (uint64_t)(nb * 2 * row));
        default: return range(s.open, (uint64_t)(4 * kKvbBlock * row));
    }
}
Range part(const kvb_seq& s, int which, int32_t kv_heads, int32_t d) {
    return part(s, which, which == SCALES ? kv_heads : (int64_t)kv_heads * d);
}

// Pointers of the parts of a sequence that a call uses (bit i of `need`: part i
// must be there; NULL bounds are allowed where they are not needed).
int check_parts(const kvb_seq& s, unsigned need) {
    const void* const ptr[PARTS] = {s.k, s.v, s.scales, s.bounds, s.open};
    for (int i = 0; i < PARTS; ++i)
        if ((need >> i & 1) && !ptr[i]) return CAP_E_INVAL;
    return CAP_OK;
}
int check_align(const kvb_seq& s) {
    return ((addr(s.k) | addr(s.v) | addr(s.bounds) | addr(s.open)) & 15) || (addr(s.scales) & 3) ? CAP_E_ALIGN : CAP_OK;
}

// Whether every part that a call uses ends below the last address.
int check_ends(const kvb_seq& s, unsigned used, int32_t kv_heads, int32_t d) {
    for (int i = 0; i < PARTS; ++i)
        if ((used >> i & 1) && wraps(part(s, i, kv_heads, d))) return CAP_E_SIZE;
    return CAP_OK;
}

// Whether an output meets one of the parts `used` of a sequence.
bool meets_cache(const Range& out, const kvb_seq& s, unsigned used, int32_t kv_heads, int32_t d) {
    for (int i = 0; i < PARTS; ++i)
        if ((used >> i & 1) && meet(out, part(s, i, kv_heads, d))) return true;
    return false;
}

constexpr unsigned bit(int i) { return 1u << i; }

// ---- attend: the launch plan ----
// Sequences of few blocks stay whole: 256 channels, runs of 2 blocks and their join 8.8 + 4.9
// us, 8 blocks whole 11.5; a pass at 200 rows of 64 channels 10.8 us cut, 6.8 whole.
constexpr int64_t kWholeBlocks = 8;

// Blocks that a run of a cut sequence takes, for tiles of 16 rows; `total`: the
// blocks of all tiles, each with its sequence's (512 tokens of 1024, 256 channels, 512 tiles
// that see 12 of 16 blocks in the mean: 27 us whole, 42 as two runs).  A workgroup to a CU while runs stay short, two where they
// are long enough for one's loads to cover the other's arithmetic.  Measured (us,
// both launches, 8 query heads on each KV head of 256; runs of): 16385 rows x 4 heads
// 2: 19.3, 4: 16.4, 6: 15.6, 8: 16.7, 16: 20.8; 131072 + 18561 rows x 4 heads
// 8: 66, 12: 67, 16: 63, 24: 72; 32 sequences of 816 rows x 1 head 2: 13.2, 4: 14.4,
// 8: 16.0, whole (13, no second launch) 15.6.
int64_t run_of_16(int64_t total, int64_t longest) {
    if (longest <= kWholeBlocks) return longest;
    const int64_t one = (total + 255) / 256;
    return std::max<int64_t>(2, one <= 16 ? one : (total + 511) / 512);
}

// What the sequences of a launch have: blocks of the longest, blocks of all tiles, those
// that they see, rows, tiles.
struct Work { int64_t longest, total, seen, rows, tiles; };

// The same for tiles of 128 rows: the length whose estimate is lowest.  A workgroup takes 5 us
// to begin and end and `alone` us a block by itself on a CU; where two fit, they take `both` us
// for a block each.  Joining takes 3 us, the runs' parts 3 TB/s.  Measured (us, both
// launches; cut into 1, 2, 3, 4, 5, 6, 8): 161 tokens behind 16384, 32 heads on 4 of 256
// channels 459, 247, 174, 138, 120, 186 (a second round), 155; of 128 355, 189, 133, 104, 87,
// 104, 86; a whole prefill of 2048 tokens, 16 heads on 4 of 128 channels 55, 59, 50, 68, 58,
// 61, 87; of 1024 30, 29, 32, 32, 32, 29, 44; of 8192 372, 468, 376.
constexpr int64_t kMostParts = 1024;
struct Plan128 { int64_t run; double us; };
Plan128 plan_128(int32_t d, const Work& x) {
    const double alone = d == 256 ? 1.75 : d == 128 ? 1.37 : 1.15, both = d == 128 ? 2.5 : 1.85, ends = 5.0;
    const double tiles = (double)x.tiles, mid = (double)x.seen / tiles;
    Plan128 best{x.longest, 1e30};
    for (int64_t cut = 1; cut <= 32 && cut <= x.longest; ++cut) {
        // (1024 parts at most bound the workspace, at 135 MB of 256 channels.  Of nine calls that would
        // take more, eight took 4 to 14 % less without the limit and one 14 % more.)
        if (cut > 1 && (x.longest <= kWholeBlocks || x.tiles * cut > kMostParts)) break;
        const int64_t run = (x.longest + cut - 1) / cut;
        // the tiles' blocks are taken as spread evenly about their mean, up to the longest: the
        // share of tiles with more than one run, and how many runs there are
        const double low = std::max(1.0, 2.0 * mid - (double)x.longest);
        const double share = run >= x.longest ? 0.0 : (double)run <= low ? 1.0 : (double)(x.longest - run) / ((double)x.longest - low);
        const double wgs = cut == 1 ? tiles : std::ceil(tiles * (mid / (double)run + 0.5 * share));
        const double mean = (double)x.seen / wgs;
        double us = alone * (double)run + ends;
        if (wgs > 256) us = std::max(us, std::ceil(wgs / (d == 256 ? 256 : 512)) * ((d == 256 ? alone : both) * mean + ends));
        if (cut > 1) us += 3.0 + (wgs - tiles * (1.0 - share)) * (double)x.rows / tiles * (double)d * 8.0 / 3e6;
        if (us < best.us) best = {run, us};
    }
    return best;
}

// Query rows of a sequence and KV head from which it may take tiles of 128 (with a block list
// never), and what tiles of 16 take instead: a time for each block and tile, more of it where
// less than a workgroup to a CU leaves them in runs, and a join.  Both launches' estimates are
// without their 4 us from call to call.  Measured (us, tiles of 16 / of 128; tokens, rows held,
// query heads on KV heads of d channels):
//     512 of 512, 16 on 4 of 256        16 / 25      16 such sequences     169 / 92
//     2048 of 2048, 16 on 4 of 256      90 / 70      of 128  55 / 46       of 64  29 / 37
//     161 behind 16384, 4 on 4 of 256   54 / 38      of 128  35 / 27       of 64  21 / 22
//     64 of 300, 16 on 4 of 256         10 / 19      32 such sequences      47 / 26
//     8192 of 8192, 16 on 4 of 256    1181 / 573     of 128 701 / 321      of 64 334 / 239
// Over 135 such calls the estimates' choice is 0.3 % behind the better one (30 % at 2048 of 2048
// of 64 channels, the worst), tiles of 128 throughout 34 %.  A tile of 128 for 64 rows takes 110 where tiles of 16 take 60 (131072 rows).
constexpr int64_t kRowsFor128 = 129;
double us_of_16(int32_t d, const Work& x) {
    const double block = d == 256 ? 2.3e-3 : d == 128 ? 1.4e-3 : 0.72e-3, tile = d == 256 ? 10e-3 : d == 128 ? 4.2e-3 : 2.6e-3;
    return 4.0 + block * (double)x.seen * (x.tiles < 256 ? 1.6 : 1.0) + tile * (double)x.tiles +
           (run_of_16(x.total, x.longest) < x.longest ? 4.0 : 0.0);
}

// p[0]: the sequences in tiles of 16 rows, p[1]: those in tiles of 128, a launch each.
int plan_attend(const kvb_attend_args* a, cap::KvbAttendParams (&p)[2]) {
    const int rc = check_sizes(a->seqs, a->n_seq, a->heads, a->kv_heads, a->d, a->in_dtype, a->tokens);
    if (rc != CAP_OK) return rc;
    if (a->idx ? a->n_sel < 1 : a->n_sel != 0) return CAP_E_INVAL;
    const int64_t G = a->heads / a->kv_heads;
    auto blocks = [&](const kvb_seq& s) { return a->idx ? (int64_t)a->n_sel : (s.n + kKvbBlock - 1) / kKvbBlock; };
    auto tiles = [&](const kvb_seq& s, int k) {  // of all KV heads
        const int64_t tile = k ? 128 : 16;
        return (a->idx ? s.T * ((G + 15) / 16) : (s.T * G + tile - 1) / tile) * a->kv_heads;
    };
    auto add = [&](Work& x, const kvb_seq& s, int k) {
        x.longest = std::max(x.longest, blocks(s));
        x.total += tiles(s, k) * blocks(s);
        x.seen += tiles(s, k) * (blocks(s) - (a->idx ? 0 : s.T / kKvbBlock / 2));  // a prefill's tiles see half of its own
        x.rows += s.T * a->heads;
        x.tiles += tiles(s, k);
    };
    auto many = [&](const kvb_seq& s) { return !a->idx && s.T * G >= kRowsFor128; };
    Work as[2] = {}, work[2] = {};  // the sequences of many rows, were they in tiles of 16 or 128; each launch
    for (int32_t i = 0; i < a->n_seq; ++i)
        for (int k = 0; k < 2 && many(a->seqs[i]); ++k) add(as[k], a->seqs[i], k);
    const bool wide = as[1].tiles > 0 && plan_128(a->d, as[1]).us < us_of_16(a->d, as[0]);
    auto kind = [&](const kvb_seq& s) { return wide && many(s) ? 1 : 0; };
    for (int32_t i = 0; i < a->n_seq; ++i)
        if (a->seqs[i].T > 0) add(work[kind(a->seqs[i])], a->seqs[i], kind(a->seqs[i]));
    int64_t per[2];
    for (int k = 0; k < 2; ++k) {
        p[k].tokens = a->tokens;
        p[k].heads = a->heads;
        p[k].kv_heads = a->kv_heads;
        p[k].d = a->d;
        p[k].n_sel = a->n_sel;
        p[k].tile = k ? 128 : 16;
        per[k] = k == 0 ? run_of_16(work[k].total, work[k].longest) : work[k].tiles > 0 ? plan_128(a->d, work[k]).run : 1;
        if (a->idx) per[k] = std::min<int64_t>(per[k], cap::kKvbListRun);
    }
    int64_t wgs[2] = {}, slots[2] = {}, t0 = 0;
    for (int32_t i = 0; i < a->n_seq; ++i) {
        const kvb_seq& s = a->seqs[i];
        if (s.T == 0) continue;
        const int k = kind(s);
        cap::KvbAttendSeq& x = p[k].seq[p[k].n_seq++];
        x.k = addr(s.k);
        x.v = addr(s.v);
        x.scales = addr(s.scales);
        x.n = s.n;
        x.t0 = t0;
        x.T = (int32_t)s.T;
        const int64_t nb = blocks(s);
        x.nsplit = (int32_t)((nb + per[k] - 1) / per[k]);
        x.per = (int32_t)((nb + x.nsplit - 1) / x.nsplit);  // of even lengths
        x.first_wg = (uint32_t)wgs[k];
        x.first_slot = (uint32_t)slots[k];
        wgs[k] += tiles(s, k) * x.nsplit;
        if (x.nsplit > 1) slots[k] += tiles(s, k) * x.nsplit;
        if (wgs[k] > 0x7fffffff) return CAP_E_UNSUPPORTED;
        t0 += s.T;
    }
    for (int k = 0; k < 2; ++k) {
        p[k].wgs = (uint32_t)wgs[k];
        p[k].slots = (uint32_t)slots[k];
    }
    return CAP_OK;
}

uint64_t attend_workspace(const cap::KvbAttendParams& p) {
    return (uint64_t)p.slots * (uint64_t)p.tile * ((uint64_t)p.d + 2) * 4;
}

// ---- select: the launch plan ----
int plan_select(const kvb_select_args* a, cap::KvbSelectParams* p, uint64_t* bytes) {
    const int64_t tokens = a->tokens;
    const int rc = check_sizes(a->seqs, a->n_seq, a->heads, a->kv_heads, a->d, a->in_dtype, tokens);
    if (rc != CAP_OK) return rc;
    if (a->first < 0 || a->last < 1 || a->n_sel < 1 || (int64_t)a->first + a->last > a->n_sel) return CAP_E_INVAL;
    uint64_t keys = 0;
    int64_t wgs = 0, t0 = 0;
    int32_t n = 0;
    for (int32_t i = 0; i < a->n_seq; ++i) {
        const kvb_seq& s = a->seqs[i];
        if (s.T == 0) continue;
        const int64_t nb = (s.n + kKvbBlock - 1) / kKvbBlock, pairs = s.T * a->kv_heads;
        cap::KvbSelectSeq& x = p->seq[n++];
        x.scales = addr(s.scales);
        x.bounds = addr(s.bounds);
        x.n = s.n;
        x.t0 = t0;
        x.T = (int32_t)s.T;
        x.first_wg = (uint32_t)wgs;
        x.keys = keys;
        keys += (uint64_t)(pairs * nb);
        wgs += pairs * ((nb + cap::kKvbScoreBlocks - 1) / cap::kKvbScoreBlocks);
        if (wgs > 0x7fffffff) return CAP_E_UNSUPPORTED;
        t0 += s.T;
    }
    p->tokens = tokens;
    p->n_seq = n;
    p->heads = a->heads;
    p->kv_heads = a->kv_heads;
    p->d = a->d;
    p->n_sel = a->n_sel;
    p->first = a->first;
    p->last = a->last;
    p->wgs = (uint32_t)wgs;
    *bytes = up(keys * 8, 16);
    return CAP_OK;
}

int launch_status(hipError_t e) { return e == hipSuccess ? CAP_OK : CAP_E_HIP; }

}  // namespace

extern "C" {

int kvb_append(const kvb_append_args* a, void* stream) {
    if (!a) return CAP_E_INVAL;
    const int64_t tokens = a->tokens;
    int rc = check_sizes(a->seqs, a->n_seq, a->kv_heads, a->kv_heads, a->d, a->in_dtype, tokens);
    if (rc != CAP_OK) return rc;
    const int64_t row = (int64_t)a->kv_heads * a->d;
    cap::KvbAppendParams p{};
    if ((rc = check_stride(a->k_stride, row, &p.k_stride)) != CAP_OK) return rc;
    if ((rc = check_stride(a->v_stride, row, &p.v_stride)) != CAP_OK) return rc;
    if (tokens == 0) return CAP_OK;
    if (!a->k || !a->v) return CAP_E_INVAL;
    const Range in[2] = {range(a->k, span(tokens, p.k_stride, row)), range(a->v, span(tokens, p.v_stride, row))};
    if (wraps(in[0]) || wraps(in[1])) return CAP_E_SIZE;
    Range out[KVB_MAX_SEQ * PARTS];
    int n_out = 0, n = 0;
    int64_t wgs = 0, t0 = 0;
    for (int32_t i = 0; i < a->n_seq; ++i) {
        const kvb_seq& s = a->seqs[i];
        if (s.T == 0) continue;
        if ((rc = check_parts(s, bit(K) | bit(V) | bit(SCALES) | bit(OPEN))) != CAP_OK) return rc;
        if ((rc = check_align(s)) != CAP_OK) return rc;
        if ((rc = check_ends(s, ~0u, a->kv_heads, a->d)) != CAP_OK) return rc;
        cap::KvbAppendSeq& x = p.seq[n++];
        x = {addr(s.k), addr(s.v), addr(s.scales), addr(s.bounds), addr(s.open), s.n, t0, (int32_t)s.T, (uint32_t)wgs};
        const int64_t begun = (s.n + kKvbBlock - 1) / kKvbBlock - (s.n - s.T) / kKvbBlock;
        wgs += begun * a->kv_heads * 2;
        if (wgs > 0x7fffffff) return CAP_E_UNSUPPORTED;
        t0 += s.T;
    }
    for (int j = 0; j < PARTS; ++j)  // in the order in which they mostly lie in memory
        for (int32_t i = 0; i < a->n_seq; ++i) {
            const Range r = part(a->seqs[i], j, a->kv_heads, a->d);
            if (a->seqs[i].T == 0 || r.a == r.b) continue;
            if (meet(r, in[0]) || meet(r, in[1])) return CAP_E_INVAL;
            out[n_out++] = r;
        }
    if ((addr(a->k) | addr(a->v)) & 15) return CAP_E_ALIGN;
    const auto lower = [](const Range& x, const Range& y) { return x.a < y.a; };
    if (!std::is_sorted(out, out + n_out, lower)) std::sort(out, out + n_out, lower);
    for (int i = 1; i < n_out; ++i)
        if (out[i].a < out[i - 1].b) return CAP_E_INVAL;
    p.k_new = a->k;
    p.v_new = a->v;
    p.n_seq = n;
    p.kv_heads = a->kv_heads;
    p.d = a->d;
    p.wgs = (uint32_t)wgs;
    return launch_status(cap::launch_kvb_append(p, static_cast<hipStream_t>(stream)));
}

uint64_t kvb_attend_workspace_bytes(const kvb_attend_args* a) {
    cap::KvbAttendParams p[2]{};
    return a && plan_attend(a, p) == CAP_OK ? attend_workspace(p[0]) + attend_workspace(p[1]) : 0;
}

int kvb_attend(const kvb_attend_args* a, void* stream) {
    if (!a || a->reserved != 0) return CAP_E_INVAL;
    const float scale_log2 = a->scale * 1.4426950408889634f;
    if (!std::isfinite(scale_log2)) return CAP_E_INVAL;
    cap::KvbAttendParams p[2]{};
    int rc = plan_attend(a, p);
    if (rc != CAP_OK) return rc;
    const int64_t width = (int64_t)a->heads * a->d;
    int64_t q_stride = 0;
    if ((rc = check_stride(a->q_stride, width, &q_stride)) != CAP_OK) return rc;
    if (a->tokens == 0) return CAP_OK;
    if (!a->q || !a->o) return CAP_E_INVAL;
    const uint64_t need = attend_workspace(p[0]) + attend_workspace(p[1]);
    if (need && !a->workspace) return CAP_E_INVAL;
    if (a->workspace_bytes < need) return CAP_E_SIZE;
    for (int32_t i = 0; i < a->n_seq; ++i) {
        if (a->seqs[i].T == 0) continue;
        if ((rc = check_parts(a->seqs[i], bit(K) | bit(V) | bit(SCALES))) != CAP_OK) return rc;
        if ((rc = check_align(a->seqs[i])) != CAP_OK) return rc;
        if ((rc = check_ends(a->seqs[i], bit(K) | bit(V) | bit(SCALES), a->kv_heads, a->d)) != CAP_OK) return rc;
    }
    if (((addr(a->q) | addr(a->o) | (need ? addr(a->workspace) : 0)) & 15) || ((addr(a->lse) | addr(a->idx)) & 3)) return CAP_E_ALIGN;
    const uint64_t tokens = (uint64_t)a->tokens;
    const Range in[2] = {range(a->q, span(a->tokens, q_stride, width)),
                         range(a->idx, tokens * (uint64_t)a->kv_heads * (uint64_t)a->n_sel * 4)};
    const Range out[3] = {range(a->o, tokens * (uint64_t)width * 2), range(a->lse, tokens * (uint64_t)a->heads * 4),
                          range(need ? a->workspace : nullptr, need)};
    for (const Range& x : in)
        if (wraps(x)) return CAP_E_SIZE;
    for (const Range& x : out)
        if (wraps(x)) return CAP_E_SIZE;
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return CAP_E_INVAL;
        if (meet(out[i], in[0]) || meet(out[i], in[1])) return CAP_E_INVAL;
        for (int32_t j = 0; j < a->n_seq; ++j)
            if (a->seqs[j].T && meets_cache(out[i], a->seqs[j], bit(K) | bit(V) | bit(SCALES), a->kv_heads, a->d)) return CAP_E_INVAL;
    }
    float* part = static_cast<float*>(a->workspace);
    for (cap::KvbAttendParams& x : p) {
        x.q = a->q;
        x.o = a->o;
        x.lse = a->lse;
        x.idx = a->idx;
        x.q_stride = q_stride;
        x.part_o = part;
        x.part_ml = part + (uint64_t)x.slots * (uint64_t)x.tile * (uint64_t)x.d;
        part = x.part_ml + (uint64_t)x.slots * (uint64_t)x.tile * 2;
        x.scale_log2 = scale_log2;
        if ((rc = launch_status(cap::launch_kvb_attend(x, static_cast<hipStream_t>(stream)))) != CAP_OK) return rc;
    }
    return CAP_OK;
}

uint64_t kvb_select_workspace_bytes(const kvb_select_args* a) {
    cap::KvbSelectParams p{};
    uint64_t bytes = 0;
    return a && plan_select(a, &p, &bytes) == CAP_OK ? bytes : 0;
}

int kvb_select(const kvb_select_args* a, void* stream) {
    if (!a) return CAP_E_INVAL;
    cap::KvbSelectParams p{};
    uint64_t need = 0;
    int rc = plan_select(a, &p, &need);
    if (rc != CAP_OK) return rc;
    const int64_t width = (int64_t)a->heads * a->d;
    if ((rc = check_stride(a->q_stride, width, &p.q_stride)) != CAP_OK) return rc;
    if (p.tokens == 0) return CAP_OK;
    if (!a->q || !a->idx || !a->workspace) return CAP_E_INVAL;
    if (a->workspace_bytes < need) return CAP_E_SIZE;
    for (int32_t i = 0; i < a->n_seq; ++i) {
        if (a->seqs[i].T == 0) continue;
        if ((rc = check_parts(a->seqs[i], bit(SCALES) | bit(BOUNDS))) != CAP_OK) return rc;
        if ((rc = check_align(a->seqs[i])) != CAP_OK) return rc;
        if ((rc = check_ends(a->seqs[i], bit(SCALES) | bit(BOUNDS), a->kv_heads, a->d)) != CAP_OK) return rc;
    }
    if (((addr(a->q) | addr(a->workspace)) & 15) || (addr(a->idx) & 3)) return CAP_E_ALIGN;
    const Range q = range(a->q, span(p.tokens, p.q_stride, width));
    const Range out[2] = {range(a->idx, (uint64_t)p.tokens * (uint64_t)a->kv_heads * (uint64_t)a->n_sel * 4), range(a->workspace, need)};
    if (wraps(q) || wraps(out[0]) || wraps(out[1])) return CAP_E_SIZE;
    if (meet(out[0], out[1]) || meet(out[0], q) || meet(out[1], q)) return CAP_E_INVAL;
    for (int i = 0; i < 2; ++i)
        for (int32_t j = 0; j < a->n_seq; ++j)
            if (a->seqs[j].T && meets_cache(out[i], a->seqs[j], bit(SCALES) | bit(BOUNDS), a->kv_heads, a->d)) return CAP_E_INVAL;
    p.q = a->q;
    p.idx = a->idx;
    p.keys = static_cast<uint64_t*>(a->workspace);
    return launch_status(cap::launch_kvb_select(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
