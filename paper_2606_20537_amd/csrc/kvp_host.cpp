// Host side of the norm and rotation of queries and keys and of the paged bf16 KV
// cache: argument checks and launches of qk_norm_rope, kvp_append and kvp_attend.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kvp.h"

namespace {

constexpr int64_t kMostStride = (int64_t)1 << 30;

uint64_t addr(const void* p) { return (uint64_t)(uintptr_t)p; }

// `count` pieces of `width` bytes, `step` bytes apart, from `a` on: the tokens of a packed tensor, the pages of a
// pool, or (count 1) a plain array.  A token's pieces are its heads, of `head` bytes, `head_step` apart.
struct Span {
    uint64_t a = 0, width = 0, step = 0, count = 0, head = 0, head_step = 0;
    bool empty() const { return a == 0 || width == 0 || count == 0; }
    uint64_t bytes() const { return empty() ? 0 : (count - 1) * step + width; }
    bool wraps() const { return a + bytes() < a; }
    bool same(const Span& x) const { return a == x.a && width == x.width && (step == x.step || count == 1) && count == x.count; }
};
Span plain(const void* p, uint64_t bytes) { return {addr(p), bytes, 0, 1, 0, 0}; }

bool meet(const Span& x, const Span& y) {
    if (x.empty() || y.empty() || x.a >= y.a + y.bytes() || y.a >= x.a + x.bytes()) return false;
    // heads of one step, of which tokens are whole ones apart: heads of several tensors in turn
    if (x.head && x.head_step == y.head_step && (x.count == 1 || x.step % x.head_step == 0) && (y.count == 1 || y.step % x.head_step == 0)) {
        const uint64_t s = x.head_step, d = y.a >= x.a ? (y.a - x.a) % s : (s - (x.a - y.a) % s) % s;
        if (d >= x.head && d + y.head <= s) return false;
    }
    if (x.count == 1 || y.count == 1 || x.step != y.step) return true;
    // pieces of one step: slices of one larger tensor, beside each other in each of its tokens
    const uint64_t d = y.a >= x.a ? (y.a - x.a) % x.step : (x.step - (x.a - y.a) % x.step) % x.step;
    return d < x.width || d + y.width > x.step;
}

// A tensor [tokens, heads, d] of `size`-byte elements: strides in bytes, and what it covers.
int check_rows(const qk_rows& r, int64_t tokens, int32_t heads, int32_t d, int size, cap::QkRows* out, Span* span) {
    int64_t head = r.head_stride, token = r.token_stride;
    if (head == 0) head = d;
    if (head < d) return CAP_E_INVAL;
    if (head > kMostStride) return CAP_E_UNSUPPORTED;
    const int64_t width = (int64_t)(heads - 1) * head + d;
    if (token == 0) token = (int64_t)heads * head;
    if (token < width) return CAP_E_INVAL;
    if (token > kMostStride) return CAP_E_UNSUPPORTED;
    if ((head | token) % 8 != 0) return CAP_E_ALIGN;
    *out = {addr(r.p), token * size, head * size};
    *span = {addr(r.p), (uint64_t)width * size, (uint64_t)token * size, (uint64_t)tokens, (uint64_t)d * size, (uint64_t)head * size};
    return CAP_OK;
}

int check_rule(const qk_rule* r, int32_t d) {
    if (r->flags & ~(QK_NORM | QK_PAIRS)) return CAP_E_INVAL;
    if (r->rot < 0 || r->axes < 0 || (r->rot > 0 && (r->axes < 1 || !r->freqs))) return CAP_E_INVAL;
    if (r->rot % 16 != 0 || r->rot > d || r->axes > 8) return CAP_E_UNSUPPORTED;
    if (r->w_dtype != CAP_DTYPE_BF16 && r->w_dtype != CAP_DTYPE_F32) return CAP_E_INVAL;
    if ((r->flags & QK_NORM) && !(std::isfinite(r->eps) && r->eps >= 1e-20f && std::isfinite(r->w_add))) return CAP_E_INVAL;
    if ((addr(r->freqs) & 7) || ((addr(r->wq) | addr(r->wk)) & 15)) return CAP_E_ALIGN;
    return CAP_OK;
}

void enter_rule(const qk_rule* r, cap::QkParams* p) {
    p->norm = r->flags & QK_NORM;
    p->pairs = r->flags & QK_PAIRS;
    p->w_f32 = r->w_dtype == CAP_DTYPE_F32;
    p->freqs = r->freqs;
    p->wq = r->wq;
    p->wk = r->wk;
    p->rot = r->rot;
    p->axes = r->rot ? r->axes : 0;
    p->eps = r->eps;
    p->w_add = r->w_add;
}

// What a rule's call reads besides the tokens.
constexpr int kRuleSpans = 4;
void rule_spans(const qk_rule* r, const int32_t* pos, int64_t tokens, int32_t d, Span* out) {
    const uint64_t w = (r->flags & QK_NORM) ? (uint64_t)d * (r->w_dtype == CAP_DTYPE_F32 ? 4 : 2) : 0;
    out[0] = plain(r->freqs, (uint64_t)r->axes * (uint64_t)r->rot * 4);
    out[1] = plain(r->wq, w);
    out[2] = plain(r->wk, w);
    out[3] = plain(pos, r->rot ? (uint64_t)tokens * (uint64_t)r->axes * 4 : 0);
}

// Sizes of a call, all of whose tokens have `rows` rows.
int32_t tokens_of_wg(int64_t tokens, int64_t rows, int32_t d);
void enter_sizes(int64_t tokens, int32_t heads, int32_t kv_heads, int64_t rows, int32_t d, cap::QkParams* p) {
    p->tokens = tokens;
    p->heads = heads;
    p->kv_heads = kv_heads;
    p->d = d;
    p->inv_d = 1.0f / (float)d;
    p->by_rows = cap::divisor((uint32_t)rows);
    p->tokens_wg = tokens_of_wg(tokens, rows, d);
}

// Tokens of a workgroup: one lot of sines serves all heads of a token, so a workgroup has whole tokens, up to five rounds
// of its 256 threads, and more of them as long as half of the places on the chip (six workgroups to a CU, 1536) have one.
// Measured (us; 1, 2, 4 and 8 tokens), 9 heads of 256: 1500 tokens 6.1, 6.1, 6.9 and 8.5; 2000 7.4, 6.5, 7.0 and 8.5; 3000 9.0, 7.5, 7.5 and
// 9.2; 4000 10.8, 9.2, 8.1 and 9.3; 6000 15.5, 12.4, 10.4 and 11.1; 8000 21.7, 18.2, 16.4 and 15.1.  40 heads of 128: 1500 7.6, 7.8, 9.6
// and 14; 2000 9.3, 8.5, 9.6 and 16; 3000 12.9, 11.7, 12.3 and 17; 4000 19.3, 17.4, 16.0 and 18.  36 heads of 256, 16384 tokens: 111, 105, 109
// and 125.  (Over 99 calls of 1000 to 16384 tokens 2.6 % behind the best of the four in the mean; for 1024 workgroups in place
// of 768 4.9 %.)
constexpr int64_t kHalfOfPlaces = 768;
int32_t tokens_of_wg(int64_t tokens, int64_t rows, int32_t d) {
    int64_t n = 1, lanes = 1;
    while (lanes < d / 16) lanes *= 2;
    while (n < cap::kQkTokens && 2 * n * rows * lanes <= 1280 && 2 * n * kHalfOfPlaces <= tokens) n *= 2;
    return (int32_t)n;
}

int check_cache(const kvp_cache* c, cap::KvpPages* g, Span (&span)[3]) {
    if (!c || c->reserved != 0) return CAP_E_INVAL;
    if (c->pages < 0 || c->page < 1 || c->columns < 1 || c->n_seq < 0 || c->kv_heads < 1 || c->d < 1) return CAP_E_INVAL;
    if (c->d != 64 && c->d != 128 && c->d != 256) return CAP_E_UNSUPPORTED;
    if (c->page % 16 != 0 || c->n_seq > KVP_MAX_SEQ || c->pages > 0x7fffffff) return CAP_E_UNSUPPORTED;
    const int64_t row = (int64_t)c->kv_heads * c->d, capacity = (int64_t)c->columns * c->page;
    if (row > 0x7fffffff / 32 || capacity > (int64_t)1 << 24) return CAP_E_UNSUPPORTED;
    const int64_t width = row * c->page, stride = c->page_stride ? c->page_stride : width;
    const int64_t columns = c->table_stride ? c->table_stride : c->columns;
    if (stride < width || columns < c->columns) return CAP_E_INVAL;
    if (stride > (int64_t)1 << 40 || columns > kMostStride) return CAP_E_UNSUPPORTED;
    if (c->n_seq > 0 && !c->table) return CAP_E_INVAL;
    if (c->pages > 0 && (!c->k || !c->v)) return CAP_E_INVAL;
    if (stride % 8 != 0 || ((addr(c->k) | addr(c->v)) & 15) || (addr(c->table) & 3)) return CAP_E_ALIGN;
    if (c->pages > 0 && (uint64_t)stride * 2 > UINT64_MAX / (uint64_t)c->pages) return CAP_E_SIZE;
    *g = {addr(c->k), addr(c->v), c->table, nullptr, nullptr, columns, stride * 2, (int32_t)c->pages, c->page, c->columns, c->n_seq,
          c->kv_heads, (int32_t)capacity, cap::divisor((uint32_t)c->page)};
    span[0] = {addr(c->k), (uint64_t)width * 2, (uint64_t)stride * 2, (uint64_t)c->pages, 0, 0};
    span[1] = {addr(c->v), (uint64_t)width * 2, (uint64_t)stride * 2, (uint64_t)c->pages, 0, 0};
    span[2] = {addr(c->table), (uint64_t)c->columns * 4, (uint64_t)columns * 4, (uint64_t)c->n_seq, 0, 0};
    for (const Span& x : span)
        if (x.wraps()) return CAP_E_SIZE;
    return CAP_OK;
}

int check_step(const int32_t* lens, const int32_t* tok0, int64_t tokens, int32_t heads, cap::KvpPages* g, Span (&span)[2]) {
    if (tokens < 0 || heads < 0) return CAP_E_INVAL;
    if (tokens > 0x7fffffff / (heads > g->kv_heads ? heads : g->kv_heads) / 3) return CAP_E_UNSUPPORTED;
    if (!tok0 && tokens != g->n_seq) return CAP_E_INVAL;
    if (g->n_seq > 0 && tokens > 0 && !lens) return CAP_E_INVAL;
    if ((addr(lens) | addr(tok0)) & 3) return CAP_E_ALIGN;
    g->lens = lens;
    g->tok0 = tok0;
    span[0] = plain(lens, (uint64_t)g->n_seq * 4);
    span[1] = plain(tok0, (uint64_t)(g->n_seq + 1) * 4);
    return span[0].wraps() || span[1].wraps() ? CAP_E_SIZE : CAP_OK;
}

// Each output apart from the others and from what is read, except from the input that it may be (own[i], or null).
int check_apart(const Span* out, const Span* const* own, int n_out, const Span* in, int n_in) {
    for (int i = 0; i < n_out; ++i)
        if (out[i].wraps()) return CAP_E_SIZE;
    for (int i = 0; i < n_in; ++i)
        if (in[i].wraps()) return CAP_E_SIZE;
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return CAP_E_INVAL;
        for (int j = 0; j < n_in; ++j)
            if (&in[j] == own[i] && out[i].same(in[j])) continue;
            else if (meet(out[i], in[j])) return CAP_E_INVAL;
    }
    return CAP_OK;
}

// ---- attend: the launch ----
// Workgroups: as many as fit the chip at once, of which a CU has one, two or four: a unit of K and one of V to each of
// four waves are 128 KiB of LDS with 256 channels, half of it with 128 (tiles of 32 rows of 64 channels: three, for their registers).
int64_t wgs_of(int32_t d, int32_t tile) { return d == 64 && tile > 16 ? 768 : 65536 / d; }

// Units that the beginning of a segment counts for: 4 to 6 us of lookups, first loads and sums, which are more units where
// these are short.  Measured (us, for 2, 4, 6, 8 and 10 units): 35 sequences of 29300^(i / 34) rows x 4 KV heads, 256 channels 142, 97,
// 86, 85 and 85, 128 channels 65, 53, 50, 50 and 50; 50 of 12200^(i / 49) rows, six tokens, 8 KV heads, 256 channels 260, 177, 154, 159
// and 162, 128 channels 218, 154, 131, 125 and 125, 64 channels 122, 87, 75, 73 and 70.
int64_t begin_of(int32_t d) { return d == 256 ? 6 : d == 128 ? 8 : 10; }

// Rows that a segment may have where no segment is cut, which spares the second launch: few, or more where there are
// segments for every workgroup.  Lengths are on the device: these are the rows that the table has room for.  Measured (us, whole / cut;
// sequences x KV heads): 1 x 4 of 64 channels, 450 rows 8.2 / 9.2, 700 9.8 / 9.7, 800 10.1 / 9.5; of 128, 450 rows 10.0 / 9.9, 600 11.1 / 10.2, 700
// 12.1 / 10.2; of 256, 240 rows 12.0 / 13.0, 450 15.9 / 12.8; 1000 rows, 64 x 4 of 256 45 / 48, 128 x 4 of 128 43 / 47, 256 x 4 of 64 47 / 52.
int64_t whole_rows(int32_t d, int64_t segments) { return segments >= wgs_of(d, 16) ? 1024 : d == 256 ? 256 : d == 128 ? 512 : 768; }

// Query rows of a segment.  16; 32 where sequences have more than 16 of a KV head on average, and 128 where they have more than
// two tiles of 32 or so, if that leaves every workgroup a segment or some units (else more segments are worth more
// than what they read again).  Measured (us, 16 / 32 / 128; sequences of so many rows x tokens, 32 heads on 4, for 64, 128 and 256 channels):
//   8 of 16384 x 4    54 / 34 / 38    72 / 63 / 61      170 / 103 / 120
//   32 of 2048 x 5    42 / 34 / 31    79 / 49 / 49      135 / 94 / 75
//   32 of 2048 x 9    66 / 39 / 37    121 / 87 / 52     219 / 147 / 88
//   32 of 2048 x 16   65 / 64 / 42    140 / 82 / 58     357 / 197 / 94
//   1 of 16384 x 9    19 / 19 / 20    30 / 25 / 27      64 / 42 / 44
//   8 of 300 x 6, G 16  8.1 / 11 / 17   11 / 14 / 22      18 / 24 / 25
//   4 of 4000 x 16    22 / 22 / 23    49 / 32 / 30      72 / 59 / 41
//   1 of 16384 x 161  136 / 102 / 70  398 / 220 / 100   809 / 437 / 195
// and prompts of 16 heads on 4: 1 x 512 9.8 / 11 / 29, 14 / 15 / 37, 39 / 29 / 37; 16 x 512 121 / 77 / 43, 261 / 155 / 56, 677 / 438 / 157;
// 64 of 100 rows x 32 16 / 18 / 15, 34 / 26 / 21, 93 / 68 / 27.  The rule takes the best of the three or one within 5 %, but for 64 of 100 x 32 of 64 and 128
// channels (32, 26 % behind), 32 of 2048 x 5 of 64 (32, 9 %) and 1 x 512 of 128 (32, 8 %).  What it does not know is the rows held: with a
// table for 16384 rows 8 of 300 x 6 take 14, 18 and 25 us.
int32_t tile_of(const kvp_cache& c, int64_t rows, int64_t seen) {
    auto fills = [&](int64_t tile, int64_t units) {
        const int64_t segments = std::max<int64_t>(c.n_seq, rows / tile) * c.kv_heads, wgs = wgs_of(c.d, (int32_t)tile);
        return segments >= wgs || segments * (seen / cap::kKvpUnit) >= units * wgs;
    };
    if (rows > (c.d == 256 ? 32 : c.d == 128 ? 64 : 96) * c.n_seq && fills(128, 6)) return 128;
    return rows > 16 * c.n_seq && fills(32, 8) ? 32 : 16;
}

int plan_attend(const kvp_attend_args* a, cap::KvpAttendParams* p, Span (&cache)[3], Span (&step)[2]) {
    int rc = check_cache(a->cache, &p->pages, cache);
    if (rc != CAP_OK) return rc;
    if ((rc = check_step(a->lens, a->tok0, a->tokens, a->heads, &p->pages, step)) != CAP_OK) return rc;
    const kvp_cache& c = *a->cache;
    if (a->heads < 1 || a->heads % c.kv_heads != 0 || a->window < 0) return CAP_E_INVAL;
    const int64_t capacity = (int64_t)c.columns * c.page, rows = a->tokens * (a->heads / c.kv_heads);
    const int64_t seen = a->window > 0 ? std::min(capacity, a->window + a->tokens) : capacity;  // rows of a segment at most
    p->whole = seen <= whole_rows(c.d, (int64_t)c.n_seq * c.kv_heads);
    p->tile = tile_of(c, rows, seen);
    // segments at most, and units of all of them (a window's rows may begin and end inside one), which the kernel counts in 32 bits
    const int64_t segments = (rows / p->tile + c.n_seq) * c.kv_heads, begin = begin_of(c.d);
    const int64_t units = std::min((capacity + cap::kKvpUnit - 1) / cap::kKvpUnit, seen / cap::kKvpUnit + 2) + begin;
    if (segments > 0x7fffffff / units) return CAP_E_UNSUPPORTED;
    p->tokens = a->tokens;
    p->heads = a->heads;
    p->d = c.d;
    p->window = a->window;
    p->by_group = cap::divisor((uint32_t)(a->heads / c.kv_heads));
    p->by_kv_heads = cap::divisor((uint32_t)c.kv_heads);
    p->begin = (int32_t)begin;
    const int64_t most = p->whole ? segments : segments * units;
    p->wgs = (uint32_t)std::min(most, wgs_of(c.d, p->tile));
    return CAP_OK;
}

uint64_t attend_parts(const cap::KvpAttendParams& p) { return p.whole ? 0 : (uint64_t)p.wgs * 2 * (uint64_t)p.tile; }
uint64_t attend_workspace(const cap::KvpAttendParams& p) {
    return p.whole || p.tokens == 0 ? 0 : attend_parts(p) * ((uint64_t)p.d + 2) * 4 + (uint64_t)p.tokens * (uint64_t)p.heads * 8;
}

int launch_status(hipError_t e) { return e == hipSuccess ? CAP_OK : CAP_E_HIP; }

}  // namespace

extern "C" {

int qk_fill_freqs(double base, int32_t rot, int32_t axes, const int32_t* sections, int32_t interleave, double* out) {
    if (!(base > 0.0) || !std::isfinite(base) || rot < 2 || rot % 2 != 0 || axes < 1 || !out || (!sections && axes != 1)) return CAP_E_INVAL;
    if (axes > 8) return CAP_E_UNSUPPORTED;
    const int32_t pairs = rot / 2;
    int32_t left[8];
    int64_t sum = 0;
    for (int32_t a = 0; a < axes; ++a) {
        left[a] = sections ? sections[a] : pairs;
        if (left[a] < 0) return CAP_E_INVAL;
        sum += left[a];
    }
    if (sum != pairs) return CAP_E_INVAL;
    for (int32_t i = 0; i < pairs; ++i) {
        int32_t axis = interleave ? i % axes : 0;
        if (left[axis] == 0)
            for (axis = 0; left[axis] == 0;) ++axis;
        --left[axis];
        for (int32_t a = 0; a < axes; ++a) out[(int64_t)a * pairs + i] = a == axis ? std::pow(base, -2.0 * i / rot) : 0.0;
    }
    return CAP_OK;
}

int qk_norm_rope(const qk_norm_rope_args* a, void* stream) {
    if (!a || !a->rule || a->tokens < 0 || a->heads < 0 || a->kv_heads < 0 || a->d < 1) return CAP_E_INVAL;
    if (a->dtype != CAP_DTYPE_BF16 && a->dtype != CAP_DTYPE_F32) return CAP_E_INVAL;
    if (a->d % 16 != 0 || a->d > 512) return CAP_E_UNSUPPORTED;
    const int64_t rows = (int64_t)a->heads + a->kv_heads;
    int rc = check_rule(a->rule, a->d);
    if (rc != CAP_OK) return rc;
    if (rows > 0 && a->tokens > 0x7fffffff / rows) return CAP_E_UNSUPPORTED;
    if (a->tokens == 0 || rows == 0) return CAP_OK;
    const int size = a->dtype == CAP_DTYPE_F32 ? 4 : 2;
    cap::QkParams p{};
    Span out[2], in[2 + kRuleSpans];
    if (a->heads > 0) {
        if (!a->q.p || !a->q_out.p) return CAP_E_INVAL;
        if ((rc = check_rows(a->q, a->tokens, a->heads, a->d, size, &p.q, &in[0])) != CAP_OK) return rc;
        if ((rc = check_rows(a->q_out, a->tokens, a->heads, a->d, size, &p.q_out, &out[0])) != CAP_OK) return rc;
    }
    if (a->kv_heads > 0) {
        if (!a->k.p || !a->k_out.p) return CAP_E_INVAL;
        if ((rc = check_rows(a->k, a->tokens, a->kv_heads, a->d, size, &p.k, &in[1])) != CAP_OK) return rc;
        if ((rc = check_rows(a->k_out, a->tokens, a->kv_heads, a->d, size, &p.k_out, &out[1])) != CAP_OK) return rc;
    }
    if (a->rule->rot > 0 && !a->pos) return CAP_E_INVAL;
    if (((p.q.p | p.k.p | p.q_out.p | p.k_out.p) & 15) || (addr(a->pos) & 3)) return CAP_E_ALIGN;
    rule_spans(a->rule, a->pos, a->tokens, a->d, in + 2);
    const Span* const own[2] = {&in[0], &in[1]};
    if (a->heads > 0 && p.q_out.p == p.q.p && p.q_out.head != p.q.head) return CAP_E_INVAL;
    if (a->kv_heads > 0 && p.k_out.p == p.k.p && p.k_out.head != p.k.head) return CAP_E_INVAL;
    if ((rc = check_apart(out, own, 2, in, 2 + kRuleSpans)) != CAP_OK) return rc;
    enter_rule(a->rule, &p);
    p.pos = a->pos;
    enter_sizes(a->tokens, a->heads, a->kv_heads, rows, a->d, &p);
    return launch_status(cap::launch_qk(p, a->dtype == CAP_DTYPE_F32, false, static_cast<hipStream_t>(stream)));
}

int kvp_append(const kvp_append_args* a, void* stream) {
    if (!a || a->reserved != 0) return CAP_E_INVAL;
    cap::QkParams p{};
    Span cache[3], step[2];
    int rc = check_cache(a->cache, &p.pages, cache);
    if (rc != CAP_OK) return rc;
    if ((rc = check_step(a->lens, a->tok0, a->tokens, a->heads, &p.pages, step)) != CAP_OK) return rc;
    const kvp_cache& c = *a->cache;
    if (a->heads > 0 && !a->rule) return CAP_E_INVAL;
    if (a->rule && (rc = check_rule(a->rule, c.d)) != CAP_OK) return rc;
    if (a->tokens == 0 || c.n_seq == 0) return CAP_OK;
    if (!a->k.p || !a->v.p) return CAP_E_INVAL;
    Span out[3], in[6 + kRuleSpans];
    if ((rc = check_rows(a->k, a->tokens, c.kv_heads, c.d, 2, &p.k, &in[0])) != CAP_OK) return rc;
    if ((rc = check_rows(a->v, a->tokens, c.kv_heads, c.d, 2, &p.v, &in[1])) != CAP_OK) return rc;
    if (a->heads > 0) {
        if (!a->q.p || !a->q_out.p) return CAP_E_INVAL;
        if ((rc = check_rows(a->q, a->tokens, a->heads, c.d, 2, &p.q, &in[2])) != CAP_OK) return rc;
        if ((rc = check_rows(a->q_out, a->tokens, a->heads, c.d, 2, &p.q_out, &out[2])) != CAP_OK) return rc;
        if (p.q_out.p == p.q.p && p.q_out.head != p.q.head) return CAP_E_INVAL;
    }
    if (((p.q.p | p.k.p | p.v.p | p.q_out.p) & 15) || (addr(a->pos) & 3)) return CAP_E_ALIGN;
    out[0] = cache[0];
    out[1] = cache[1];
    in[3] = cache[2];
    in[4] = step[0];
    in[5] = step[1];
    if (a->rule) rule_spans(a->rule, a->pos, a->tokens, c.d, in + 6);
    const Span* const own[3] = {nullptr, nullptr, &in[2]};
    if ((rc = check_apart(out, own, 3, in, 6 + kRuleSpans)) != CAP_OK) return rc;
    if (a->rule) enter_rule(a->rule, &p);
    p.pos = a->pos;
    enter_sizes(a->tokens, a->heads, c.kv_heads, (int64_t)a->heads + 2 * c.kv_heads, c.d, &p);
    return launch_status(cap::launch_qk(p, false, true, static_cast<hipStream_t>(stream)));
}

uint64_t kvp_attend_workspace_bytes(const kvp_attend_args* a) {
    cap::KvpAttendParams p{};
    Span cache[3], step[2];
    if (!a) return 0;
    kvp_attend_args sizes = *a;  // (lens and tok0 do not matter)
    static const int32_t none = 0;
    sizes.lens = sizes.tok0 = &none;
    return plan_attend(&sizes, &p, cache, step) == CAP_OK ? attend_workspace(p) : 0;
}

int kvp_attend(const kvp_attend_args* a, void* stream) {
    if (!a || a->reserved != 0) return CAP_E_INVAL;
    cap::KvpAttendParams p{};
    p.scale_log2 = a->scale * 1.4426950408889634f;
    if (!std::isfinite(p.scale_log2)) return CAP_E_INVAL;
    if (p.scale_log2 == 0.0f) p.scale_log2 = 0x1p-149f;
    Span cache[3], step[2];
    int rc = plan_attend(a, &p, cache, step);
    if (rc != CAP_OK) return rc;
    if (a->tokens == 0 || a->cache->n_seq == 0) return CAP_OK;
    if (!a->q.p || !a->o) return CAP_E_INVAL;
    Span out[3], in[6] = {{}, cache[0], cache[1], cache[2], step[0], step[1]};
    if ((rc = check_rows(a->q, a->tokens, a->heads, p.d, 2, &p.q, &in[0])) != CAP_OK) return rc;
    const uint64_t need = attend_workspace(p), rows = (uint64_t)a->tokens * (uint64_t)a->heads;
    if (need && !a->workspace) return CAP_E_INVAL;
    if (a->workspace_bytes < need) return CAP_E_SIZE;
    if (((p.q.p | addr(a->o) | (need ? addr(a->workspace) : 0)) & 15) || (addr(a->lse) & 3)) return CAP_E_ALIGN;
    out[0] = plain(a->o, rows * (uint64_t)p.d * 2);
    out[1] = plain(a->lse, rows * 4);
    out[2] = plain(need ? a->workspace : nullptr, need);
    const Span* const own[3] = {};
    if ((rc = check_apart(out, own, 3, in, 6)) != CAP_OK) return rc;
    p.o = a->o;
    p.lse = a->lse;
    p.part_o = static_cast<float*>(a->workspace);
    p.part_ml = p.part_o + attend_parts(p) * (uint64_t)p.d;
    p.meta = reinterpret_cast<uint64_t*>(p.part_ml + attend_parts(p) * 2);
    return launch_status(cap::launch_kvp_attend(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
