// C ABI of the RotateK hot path: argument validation, workspace carving and
// kernel launches.  See include/rotatek.h for the contract of every entry point.
#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "rk_kernels.hpp"
#include "rotatek.h"

struct rk_ctx {
    int device;           // RK_DEVICE_NONE: host-only validation context
    int n_cu;
    int force_generic;
    int decode_splits;
    int fuse_merge;       // fold the split-K merge into the split launch where the shape allows it
    int xcd_deal_ok;      // work-groups with equal (linear index mod 8) share an XCD on this device (probed)
    int32_t* tickets;     // device: APP_TICKETS zero-initialised counters (one per batch item, rk_append)
    void* static_scratch; // this device's copy of `scratch` below (its device address), for rk_decode_attn_static
    char err[256];
};

// Split-K partials of rk_decode_attn_static, for callers that cannot hand over a workspace they
// allocated.  Every GPU the library runs on holds its own copy until the process ends.  In host code
// this name is only a stand-in for the symbol: the device address of a GPU's copy comes from
// hipGetSymbolAddress (rk_create, with that device current) and is what kernels and copies receive.
// Nothing in it has to start at zero: the merge kernel reads exactly the partial slots that the split
// kernel of the same call has written.
static __device__ __align__(256) unsigned char scratch[RK_STATIC_SCRATCH_BYTES];

namespace {

using namespace rk;

rk_status fail(rk_ctx* ctx, rk_status s, const char* fmt, ...)
{
    if (ctx) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap);
        va_end(ap);
    }
    return s;
}

rk_status hip_fail(rk_ctx* ctx, hipError_t e, const char* what)
{
    return fail(ctx, RK_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

constexpr int APP_TICKETS = CONTEXT_TICKETS;   // >= batch
constexpr int DEC_COUNTERS = 1 << 16;  // units (b, h_kv, head group) whose split-K merge can ride in the split launch

size_t elem_size(int dtype) { return dtype == RK_F32 ? 4 : 2; }
size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

rk_status check_layout(rk_ctx* ctx, const rk_layout* L)
{
    if (!L) return fail(ctx, RK_ERR_INVALID_ARG, "layout is NULL");
    if (L->head_dim != D) return fail(ctx, RK_ERR_UNSUPPORTED, "head_dim %d: only 128 is supported", L->head_dim);
    if (L->dtype != RK_F32 && L->dtype != RK_BF16) return fail(ctx, RK_ERR_UNSUPPORTED, "unknown dtype %d", L->dtype);
    if (L->batch < 1 || L->n_q_heads < 1 || L->n_kv_heads < 1)
        return fail(ctx, RK_ERR_INVALID_ARG, "batch/head counts must be positive");
    if (L->batch > 65535 || L->n_q_heads > 65535) return fail(ctx, RK_ERR_INVALID_ARG, "batch/head counts exceed 65535");
    if (L->n_q_heads % L->n_kv_heads != 0)
        return fail(ctx, RK_ERR_INVALID_ARG, "n_q_heads %d is not a multiple of n_kv_heads %d", L->n_q_heads, L->n_kv_heads);
    if (L->keep < 1 || L->keep > D) return fail(ctx, RK_ERR_INVALID_ARG, "keep %d outside 1..128", L->keep);
    if (L->capacity < 32 || L->capacity % 32 != 0)
        return fail(ctx, RK_ERR_INVALID_ARG, "capacity %d must be a positive multiple of 32", L->capacity);
    if (L->max_seq_len < 0) return fail(ctx, RK_ERR_INVALID_ARG, "max_seq_len is negative");
    // token counts stay below 2^30, so that rounding one up to a tile never leaves the range of int
    if (L->capacity > RK_MAX_TOKENS || L->max_seq_len > RK_MAX_TOKENS)
        return fail(ctx, RK_ERR_INVALID_ARG, "capacity / max_seq_len exceed %d tokens", RK_MAX_TOKENS);
    return RK_OK;
}

rk_status check_rows(rk_ctx* ctx, const rk_layout* L, const rk_rows* r, const char* name)
{
    if (!r || !r->data) return fail(ctx, RK_ERR_INVALID_ARG, "%s: NULL", name);
    if (r->n_tokens < 0) return fail(ctx, RK_ERR_INVALID_ARG, "%s: n_tokens is negative", name);
    if (r->n_tokens > RK_MAX_TOKENS) return fail(ctx, RK_ERR_INVALID_ARG, "%s: n_tokens exceeds %d", name, RK_MAX_TOKENS);
    if (r->tok_idx && !r->tok_off) return fail(ctx, RK_ERR_INVALID_ARG, "%s: tok_idx given without tok_off", name);
    if (r->stride_t < D || r->stride_b < 0 || r->stride_h < 0)
        return fail(ctx, RK_ERR_INVALID_ARG, "%s: bad strides", name);
    const int64_t ea = 16 / (int64_t)elem_size(L->dtype);    // elements per 16 bytes
    if (((uintptr_t)r->data & 15) || r->stride_t % ea || r->stride_b % ea || r->stride_h % ea)
        return fail(ctx, RK_ERR_INVALID_ARG, "%s: rows must be 16-byte aligned", name);
    return RK_OK;
}

bool ranges_meet(const void* a, size_t a_bytes, const void* b, size_t b_bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + b_bytes && y < x + a_bytes;
}

RowsDev to_dev(const rk_rows* r)
{
    RowsDev d;
    d.data = r->data; d.sb = r->stride_b; d.sh = r->stride_h; d.st = r->stride_t;
    d.n_tokens = r->n_tokens; d.n_dev = r->n_tokens_dev; d.tok_idx = r->tok_idx; d.tok_off = r->tok_off;
    return d;
}

// Chunk partials the workspace holds per (b, h_kv): what any choice of kernel needs (the size is given without a
// context) for any number of rows up to max_tokens (a workspace may be reused for a shorter input, which may take shorter
// chunks).
int cov_chunks(const rk_layout* L, int max_tokens)
{
    const int n = (max_tokens + COV_CHUNK - 1) / COV_CHUNK, few = cov_short_chunks(L->dtype, (int64_t)L->batch * L->n_kv_heads);
    const int m = (max_tokens + COV_CHUNK_MIN - 1) / COV_CHUNK_MIN, k = m < few ? m : few;
    return n > k ? (n < 1 ? 1 : n) : (k < 1 ? 1 : k);
}

// The covariance partials are dead once the covariance is reduced: the eigensolver's
// scratch reuses their space (the region is sized for the larger of the two).
struct FitWs { size_t part_S, part_sum, cov, status, total; };
FitWs fit_ws(const rk_layout* L, int max_tokens)
{
    size_t U = (size_t)L->batch * L->n_kv_heads, nc = (size_t)cov_chunks(L, max_tokens);
    FitWs w;
    w.part_S = 0;
    size_t first = U * nc * D * D * sizeof(float);
    if (first < eig_scratch_bytes(U)) first = eig_scratch_bytes(U);
    w.part_sum = align_up(w.part_S + first, 256);
    w.cov = align_up(w.part_sum + U * nc * D * sizeof(float), 256);
    w.status = align_up(w.cov + U * D * D * sizeof(float), 256);
    w.total = align_up(w.status + 2 * U * sizeof(int32_t), 256);
    return w;
}

bool use_mfma_decode(const rk_ctx* ctx, const rk_layout* L)
{
    return !(ctx && ctx->force_generic) && L->keep >= 1 && L->keep <= D;
}

rk_status check_text(rk_ctx* ctx, const rk_text* t, bool need_len)
{
    if (!t->k || !t->v) return fail(ctx, RK_ERR_INVALID_ARG, "text: NULL k or v");
    if (((uintptr_t)t->k & 15) || ((uintptr_t)t->v & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "text: k and v must be 16-byte aligned");
    if (t->stride_b < 0 || t->stride_h < 0 || t->stride_t < D || (t->stride_b % 8) || (t->stride_h % 8) ||
        (t->stride_t % 8))
        return fail(ctx, RK_ERR_INVALID_ARG, "text: strides must be non-negative multiples of 8 elements, stride_t >= %d", D);
    if (t->capacity < 0 || t->max_len < 0) return fail(ctx, RK_ERR_INVALID_ARG, "text: negative capacity or max_len");
    if (t->max_len > t->capacity)
        return fail(ctx, RK_ERR_INVALID_ARG, "text: max_len %d exceeds capacity %d", t->max_len, t->capacity);
    if (need_len && !t->len) return fail(ctx, RK_ERR_INVALID_ARG, "text: len is NULL");
    return RK_OK;
}

// N_s for `units` work-groups a split; splits of at least `tiles_min` 128-token tiles on long caches
int plan_splits(const rk_ctx* ctx, long units, int tiles, int tiles_min)
{
    int S;
    if (ctx && ctx->decode_splits > 0) S = ctx->decode_splits;
    else {
        // one 4-wave work-group per compute unit: a second one gets its memory requests served only
        // after the first one's (measured: its prologue then ends 10 us later), and every work-group
        // pays its own prologue and partial
        // (rounded down: a few work-groups more than compute units would run as a second round)
        const long target = ctx ? ctx->n_cu : 256;
        S = (int)(target / units);
        if (S < 1) {
            // more units than compute units: a partly filled last round costs a whole round (320 units:
            // 186 us unsplit, 162 us with four splits); take the split count 1..4 that wastes least of it
            S = 1;
            double best = 1e30;
            for (int c = 1; c <= 4; ++c) {
                const double cost = (double)((units * c + target - 1) / target) / c;
                if (cost < best - 1e-9) { best = cost; S = c; }
            }
        }
        if (S > 64) S = 64;
        // 512 tokens to a split (256 in fp32), and under 2K tokens up to four splits of 256: what a split's prologue and partial were worth
        // when they cost 3 us more.  more_splits() goes on from here where compute units are idle.
        const int cap_long = tiles / tiles_min, cap_short = tiles / 2 < 4 ? tiles / 2 : 4;
        const int cap = cap_long > cap_short ? cap_long : cap_short;
        if (S > cap) S = cap;
    }
    if (S > tiles) S = tiles;
    return S < 1 ? 1 : S;
}

// partials: the slots per (b, h_q) whose (m, l, acc[d]) the workspace holds, plus one score per row for a fused append
size_t partial_bytes(const rk_layout* L, int slots)
{
    return align_up((size_t)L->batch * L->n_q_heads * ((size_t)slots * (D + 2) + 1) * sizeof(float), 256);
}

// Splits of a dual decode (bf16 matrix-core kernels) that take text rows alone, next to the S of the cache; 0: every split
// takes its part of the text in front of its part of the cache.
int text_splits(const rk_ctx* ctx, const rk_layout* L, int S, int text_rows)
{
    if ((ctx && ctx->decode_splits > 0) || text_rows <= 0) return 0;
    const int G = L->n_q_heads / L->n_kv_heads;
    const long units = (long)L->batch * L->n_kv_heads * ((G + 15) / 16), n_cu = ctx ? ctx->n_cu : 256;
    const long left = n_cu / units - S, room = 2 * n_cu / units - S;      // to one and to two work-groups a compute unit
    auto pieces = [&](int rows) { return (long)(((int64_t)text_rows + rows - 1) / rows); };
    auto least = [](long a, long b) { return (int)(a < b ? a : b); };
    if (left >= 1) {
        // compute units are left over: a split per 128 rows (a 32-row tile for each wave), but no more than are left ...
        if (pieces(128) <= left) return least(pieces(128), DECODE_TEXT_SPLITS_MAX);
        // ... unless each would then read more than twice what a split of the cache does: the launch waits for them
        // (32 units x 3700 tokens, S = 7, 1500 rows: 22.2 us with one, 17.3 with eight; 500 rows: 13.8 / 15.0).  Next to one split
        // a unit the text is most of the launch, and second work-groups pay later (128 x 256 tokens, 1024 rows: 16.7 us with
        // one, 17.9 with three; 1500 rows: 25.8 / 23.1).
        const double text = 512.0 * text_rows / (double)left;
        const double cache = (double)L->max_seq_len / S * 2.0 * (keep_padded(L->keep) + D);
        if (text <= (S == 1 ? 6.0 : 2.0) * cache) return least(left, DECODE_TEXT_SPLITS_MAX);
        return least(least(pieces(128), room), DECODE_TEXT_SPLITS_MAX);
    }
    // The device is full.  One split a unit: its text in a second one would be another round (256 x 4096 tokens, 64 rows: 64.8 us
    // shared, 66.9 apart).
    if (S == 1) return 0;
    const double text = 512.0 * text_rows, cache = (double)L->max_seq_len / S * 2.0 * (keep_padded(L->keep) + D);
    if (room >= 1) {
        // Long splits of the cache cover a tile of text for each wave (32 x 22417 tokens, 742 rows: 188 us for four tokens, 199 with
        // eight splits of text; 32 x 16384, 1024 rows 38.5 us a step, 45.3 in vector code as before).
        if (S >= 4 && text_rows > 128 && text_rows <= 128 * S && cache >= 400e3) return 0;
        // Else a split per 64 rows runs beside the cache's as a second work-group (32 x 8192 tokens, 200 rows: 20.5 us, shared 21.2,
        // vector code 21.6), on no more than half the compute units while both are short (128 x 864 tokens, 227 rows, four
        // tokens: 57 us with one split a unit, 65 with two, 64 shared).
        const long most = text_rows <= 128 || (cache < 400e3 && text < 2.5 * cache) ? (room + 1) / 2 : room;
        return least(least(pieces(64), most), DECODE_TEXT_SPLITS_MAX);
    }
    // several rounds: more work-groups pay while the text is short (320 x 1024 tokens, S = 4: 200 rows 33.6 us with one split, 37.1
    // shared; 1024 rows 59 / 57)
    return pieces(256) <= 2 ? (int)pieces(256) : 0;
}

// More splits than `least` (plan_splits) where units of work-groups leave compute units idle, up to `most`: the count that comes out cheapest.
//   A split's own time goes by round trips, not by tokens: with 4 waves and two tiles a wave in flight, 256 tokens of bf16 take one (1.5 us at
//   r = 64, 0.8 for 128), 128 of fp32 2.3 us; a split of text rows beside them some 2.2.  All splits together cannot be faster than the device
//   streams.  A split more is another prologue and a partial more, folded 4, 8 or 16 a round trip; none with one split.
// Measured with each count (us): bf16 8 units x 2000 tokens, r = 64: 4 splits 8.0, 6 7.8, 8 6.5, 16 7.0; 2 x 6000: 11 9.6, 16 7.7, 24 7.5, 32 7.6; 32 x
// 2944: 5 10.3, 6 9.6, 8 10.2; 32 x 1500: 4 8.0, 6 7.6, 8 7.5; 16 x 900, r = 128: 4 7.8, 8 8.0; 8 x 300, r = 32: 1 5.1, 3 5.7; with 64 text rows
// 8 x 1000, four tokens: 4 29.8, 8 31.1; fp32 8 x 1024, r = 32: 4 10.9, 8 8.6; 32 x 500, r = 64: 2 11.3, 4 9.2.
int more_splits(const rk_ctx* ctx, const rk_layout* L, long units, int tiles, int least, int most, bool f32, int text_rows)
{
    const int token_bytes = (keep_padded(L->keep) + D) * (int)elem_size(L->dtype);
    const double unit = f32 ? 2.3 * token_bytes / 768 : 1.5 * token_bytes / 384, stream = 128e-6 * units * tiles * token_bytes / 6.5;
    double best = 1e30;
    int S = least;
    for (int c = least, each; c <= most; c = each > 1 ? (tiles + each - 2) / (each - 1) : most + 1) {     // (the fewest splits of a length)
        each = (tiles + c - 1) / c;
        const int parts = c + (f32 ? 0 : text_splits(ctx, L, c, text_rows));
        double own = unit * (f32 ? each : each == 1 ? 0.55 : (each + 1) / 2);
        if (parts > c && own < 2.2) own = 2.2;
        const double fold = parts == 1 ? 0.0 : parts <= 4 ? 1.9 : parts <= 8 ? 2.1 : 1.9 + (parts + 15) / 16;
        const double cost = (own > stream ? own + 0.35 * stream : stream + 0.35 * own) + fold + 0.005 * L->keep / 64 * units * c;
        if (cost < best - 0.1) { best = cost; S = c; }
    }
    return S;
}

// N_s, the number of 128-token tiles they share (split s gets floor(tiles / N_s) tiles, the last tiles % N_s splits one
// more) and the bytes of workspace that the call asks for
struct DecodePlan { int S, tiles; size_t bytes; };
DecodePlan decode_plan(const rk_ctx* ctx, const rk_layout* L, int text_rows = 0)
{
    const int G = L->n_q_heads / L->n_kv_heads;
    const bool mfma = use_mfma_decode(ctx, L), f32 = mfma && L->dtype == RK_F32;
    const long rows = (long)L->batch * L->n_q_heads, groups = (long)L->batch * L->n_kv_heads * ((G + 15) / 16);
    DecodePlan p;
    p.tiles = ((L->max_seq_len > 0 ? L->max_seq_len : 1) + 127) / 128;
    // (fp32 rows are twice as long: splits of 256 tokens there)
    p.S = plan_splits(ctx, mfma ? groups : rows, p.tiles, f32 ? 2 : 4);
    int slots = p.S + DECODE_TEXT_SPLITS_MAX;
    if (f32) {
        // The size of an fp32 workspace is that of the plain kernel's plan (a split count per query head), by which
        // rk_decode_attn_static takes or refuses a shape: splits per KV head, up to 16 times as many, may not take it over
        // the built-in scratch.  The text takes no splits here, so all slots are the cache's.
        slots = plan_splits(ctx, rows, p.tiles, 4) + DECODE_TEXT_SPLITS_MAX;
        while (p.S > slots && partial_bytes(L, p.S) > RK_STATIC_SCRATCH_BYTES) --p.S;
        if (slots < p.S) slots = p.S;
    }
    // The splits that more_splits() adds have to fit into four times what these few need, and into the built-in scratch if these do.  A size by
    // the finer plan itself grows with every 128 tokens, so that a caller who sized once would soon hold too little (1 x 32 query heads on 8 KV heads:
    // 266 KB at 1000 tokens, 283 at 1030, 666 at 4000).  What is asked rises and falls with the coarse plan's size, whatever the shapes: a
    // workspace that serves one call by the coarse plan serves it by this one.
    p.bytes = partial_bytes(L, slots);
    if (p.bytes < RK_STATIC_SCRATCH_BYTES) p.bytes = 4 * p.bytes < RK_STATIC_SCRATCH_BYTES ? 4 * p.bytes : RK_STATIC_SCRATCH_BYTES;
    const int n_cu = ctx ? ctx->n_cu : 256;
    if (mfma && !(ctx && ctx->decode_splits > 0) && groups <= n_cu) {
        long most = ((long)(p.bytes / (sizeof(float) * rows)) - 1) / (D + 2) - (f32 ? 0 : DECODE_TEXT_SPLITS_MAX);
        if (most > n_cu / groups) most = n_cu / groups;
        if (most > 64) most = 64;
        if (most > p.tiles) most = p.tiles;
        if (most > p.S) p.S = more_splits(ctx, L, groups, p.tiles, p.S, (int)most, f32, text_rows);
    }
    return p;
}

// Attention of T query tokens a sequence: row blocks of a KV head, splits of the cache and of the full-width rows.
struct RowsPlan { int per, nrb, Sv, Sr; };
// Rows of a work-group.  16 of them leave every wave to its own tokens (attn_rows), which reads the cache once for each 16; 128 (64) share what is staged in LDS
// (attn_block; bf16 rows alone: fp32 rows would take twice the registers).  While the 16s fit beside each other on the device and the tokens are few, reading
// again from the L2 costs less than staging, waves without rows and steps behind barriers.  us with 16 / 64 / 128 rows a work-group, r = 64, bf16: 8 units x 1000
// tokens, 128 rows 13.2 / 17.3 / 17.8; 8 x 16000, 96 26.4 / 35.3 / 29.6, 128 32.7 / 37.0 / 32.2; 32 x 2000, 128 21.0 / 32.0 / 27.0; 32 x 8000, 32
// 27.4 / 38.8 / 32.0, 96 56.0 / 54.0 / 43.7; 256 x 600, 32 25.2 / 35.6 / 29.2, 64 45.9 / 42.7 / 36.6; over 8 bits: 8 x 16000, 40 21.5 / 24.3 / 31.1, 96
// 36.3 / 34.8 / 34.8; 32 x 8000, 32 24.2 / 29.0 / 33.5, 64 38.9 / 36.6 / 43.0, 128 66.4 / 55.3 / 53.2; 128 x 2000, 64 42.6 / 38.1 / 47.1, 448 - / 169.6 /
// 148.0.  (fp32 rows, 16 against 32 a work-group while there were such kernels: 8 x 16000, 32 35.6 / 41.5; 256 x 600, 32 67 / 58.5.)  Tokens of the text count as the
// cache's: 8 units, 64 rows, 1000 cached and 4000 of text 16.4 / - / 19.1, 30000 of text 46.3 / - / 40.7, over 8 bits 46.1 / 38.4 / 40.7; 32 units, 112 rows, 8000 of text
// 83.8 / - / 59.5.
int rows_per_group(const rk_ctx* ctx, const rk_layout* L, int T, int text_rows, bool q8)
{
    const int64_t rows = (int64_t)T * (L->n_q_heads / L->n_kv_heads), units = (int64_t)L->batch * L->n_kv_heads, n_cu = ctx ? ctx->n_cu : 256;
    const int64_t blocks = (rows + 15) / 16 * units;
    if (L->dtype == RK_F32 || rows <= 32 || (blocks <= 2 * n_cu && blocks * ((int64_t)L->max_seq_len + text_rows) <= 2500 * n_cu)) return 16;
    return q8 && rows <= 64 ? 64 : 128;
}
// partial slots of a row: what any length may take
int rows_slots(const rk_ctx* ctx, const rk_layout* L, int T)
{
    const int64_t rows = (int64_t)T * (L->n_q_heads / L->n_kv_heads), n_cu = ctx ? ctx->n_cu : 256;
    int64_t s = 2 * n_cu / ((rows + 127) / 128 * L->batch * L->n_kv_heads);
    s = s < 10 ? 10 : s > 64 ? 64 : s;
    if (ctx && ctx->decode_splits > 0 && s < ctx->decode_splits + 8) s = ctx->decode_splits + 8;
    return (int)s;
}
size_t rows_ws(const rk_ctx* ctx, const rk_layout* L, int T)
{
    // (256 bytes more: the accumulators begin a cache line, whatever the workspace's address)
    return align_up((size_t)L->batch * T * L->n_q_heads * rows_slots(ctx, L, T) * (D + 2) * sizeof(float), 256) + 256;
}
// The split counts whose launch comes out cheapest, in microseconds as measured: a work-group begins with some 6; a step of its loop (four waves and 32
// tokens each; of the kernels of many rows 32 tokens with 128 rows, 64 with 64) takes, at r = 64, with 16 rows bf16 0.37, fp32 1.8, 8 bits 0.67 (fp32
// rows 0.9), with many 0.72 and 1.2; a step of full-width rows 2 to 3, which is their latency.  All work-groups of few rows cannot be faster than the
// device streams; of many rows two share a compute unit and each takes half as long again.  A split more is a partial a row, written and read.  The
// splits of full-width rows come last: they run beside the others while there is room for two work-groups a compute unit (of few rows; over an fp32 cache, whose
// registers leave room for one, some 5 behind: 20 rows, 32 x 2000 tokens 29.3 with 4 splits, 26.3 with 3; 32 x 8000 57.5 and 61.1), and behind them otherwise.  Measured with each count (us): one token over 8 bits, 8 units x 30000 / 8 tokens, r = 64: 8 splits 31.0, 16 20.0, 32 15.1, 48 13.9; 16 x 8 units x
// 600, r = 128: 1 12.1, 2 13.4, 4 15.6; 32 rows, 32 x 16000: 2 64.1, 3 50.4, 4 44.1, 6 52.9, 8 46.1; 8 x 16000: 8 18.0, 12 16.4, 16 16.4, 24 18.6; 448
// rows over 8 bits, 32 x 16384: 2 291, 4 243, 6 264, 8 259.  A text that is longer than the cache decides by itself, by its bytes and its steps on a full device (splits of
// the text, the cache's at their best): one token over 8 bits, 8 units, 2880 cached, 100000 of text: 1 1378, 4 355, 8 185, 16 101, 24 74.4, 32 77.3, 60 78.4; 32 rows,
// 8 units, none cached, 30000 of text: 8 54.4, 16 33.0, 24 32.5, 32 30.2, 60 33.2; fp32 32 units, 4000 cached, 12000 of text: 1 466, 4 136, 8 99.8, 12 105; 112 rows (128 a
// work-group), 32 units, 1000 and 8000: 1 309, 4 90, 8 61.2, 12 59.5.  (The constants are for r = 64, by channels for others: of 33 shapes with r = 16, 32 and 128
// the plan came within 4 % of the best rows and splits in the middle, 19 % at worst.)
// (per: rows of a work-group, 0: the cheapest)
RowsPlan rows_plan(const rk_ctx* ctx, const rk_layout* L, int T, int text_rows, bool drafts, bool q8, int per = 0)
{
    RowsPlan p;
    p.per = per ? per : rows_per_group(ctx, L, T, text_rows, q8);
    const int64_t units = (int64_t)L->batch * L->n_kv_heads, rows = (int64_t)T * (L->n_q_heads / L->n_kv_heads);
    p.nrb = (int)((rows + p.per - 1) / p.per);
    const bool block = p.per > 16, f32 = L->dtype == RK_F32;
    const int64_t groups = p.nrb * units;
    const int n_cu = ctx ? ctx->n_cu : 256, slots = rows_slots(ctx, L, T), n_wg = block ? 2 * n_cu : n_cu;
    const int step = p.per == 128 ? 32 : p.per == 64 ? 64 : 128;
    const int nv = (L->max_seq_len + step - 1) / step;
    const int64_t text = text_rows;        // (its bound is the caller's, up to the largest int)
    const int nr = (int)(block ? (text + 63) / 64 + (drafts ? 1 : 0) : ((text + 31) / 32 + (drafts ? (T + 31) / 32 : 0) + 3) / 4);
    const double wide = (keep_padded(L->keep) + D) / 192.0;
    const double tv = wide * (p.per == 128 ? 0.72 : p.per == 64 ? 1.2 : q8 ? (f32 ? 0.9 : 0.67) : f32 ? 1.8 : 0.37);
    const double tr = block ? 3.0 : f32 ? 4.0 : 2.0;
    const double token = q8 ? keep_padded(L->keep) + D + 4 : (double)elem_size(L->dtype) * (keep_padded(L->keep) + D);
    const double stream = block ? 0.0 : (double)units * L->max_seq_len * token / 6.2e6;
    // what all full-width rows take at least, however they are split: read once, and their steps on a full device
    const double text_stream = (double)units * text * 2 * D * elem_size(L->dtype) / 6.2e6, text_steps = (double)groups * nr * (block ? 4.5 : f32 ? 4.0 : 1.3) / n_wg;
    const double least = text_stream > text_steps ? text_stream : text_steps;
    auto cost = [&](int sv, int sr) {
        const int S = sv + sr;
        const int64_t W = groups * S;
        const double shared = block && W > n_cu ? 1.5 : 1.0;
        double v = (nv + sv - 1) / sv * tv * shared, r = sr ? (nr + sr - 1) / sr * tr * shared : 0.0, behind = 0.0;
        v = v > stream ? v + 0.35 * stream : stream + 0.35 * v;
        if (sr && r < least) r = least;
        const int64_t rounds = (groups * sv + n_wg - 1) / n_wg;
        if (W > rounds * n_wg) behind = block || W > 2 * n_cu ? 6.0 + r : f32 && !q8 ? 3.0 + 0.5 * r : 0.2 * r;
        // beside the last round, and longer than it: a long text keeps the memory busy, which the cache's steps wait for too (32 units, 4000 cached and 12000 of text: 1 + 8
        // splits 53.0, 8 + 8 39.6)
        if (r > v && behind < (r - v) * (1.0 + 0.5 * v / r)) behind = (r - v) * (1.0 + 0.5 * v / r);
        const double merge = S == 1 ? 0.0 : 2.5 + S / 32.0 + (double)rows * units * S * 1040 / 5e6;
        return (6.0 + v) * rounds + behind + merge;
    };
    const int most_v = nv < 1 ? 1 : nv < 48 ? nv : 48, r0 = nr ? 1 : 0, r1 = nr < 63 && nr < slots ? nr : slots < 64 ? slots - 1 : 63;
    static const int tries[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48};
    double best = 1e30;
    p.Sv = 1;
    p.Sr = r0;
    for (int r = r0; r <= r1; r += r < 4 ? 1 : r < 8 ? 2 : r < 16 ? 4 : r < 32 ? 8 : 14) {
        auto look = [&](int64_t v) {
            if (v < 1 || v > most_v || v > slots - r) return;
            const double c = cost((int)v, r);
            if (c < best - 0.01) { best = c; p.Sv = (int)v; p.Sr = r; }
        };
        for (int v : tries) look(v);
        look(n_wg / groups - r);            // what fills the device
        look(n_wg / groups);                // without the full-width rows
    }
    if (ctx && ctx->decode_splits > 0) {
        p.Sv = ctx->decode_splits;
        if (p.Sr > slots - p.Sv) p.Sr = slots - p.Sv;         // (eight at least, see rows_slots)
    }
    return p;
}

// Text rows that one token sees at most.
int window_rows(int max_len, int window, int sinks)
{
    if (window <= 0 || window >= max_len) return max_len;
    const int64_t most = (int64_t)window + sinks;
    return most < max_len ? (int)most : max_len;
}
// One token with a window on the text.  Without a cache a split of text takes 128 rows (a tile for each wave), more where the compute units have their work-group; us, 8 units x
// 1028 rows 8 splits 9.3, 9 8.2, 16 8.0, 24 8.6; 1 x 8000 16 12.7, 32 10.1, 63 9.9; fp32 32 x 900 4 14.8, 8 12.1, 16 17.1; 256 x 4100 1 93.7, 2 96.8.
// With one, the splits of both that come out cheapest, in microseconds as fitted to 300 to 800 shapes of each kind in some 80 splits each (8 to 128 query heads, 100 to 33000 cached tokens, 50 to 12000 rows of
// text): what is begun is waited for, then the longest wave's tiles (of either) or all bytes, partials are written and folded.  Of 1079 other shapes its time was 2 % (bf16), 1 (fp32), 3 and 4 (8 bits)
// above the best of all splits on average, 22 % at worst; the plan of drafts 7, 6, 4 and 4, 34 at worst. us, that / this: 64 units, 3000 + 6000 rows 1 + 4 splits 55, 1 + 3 44; 32 units, 4000 +
// 8000 1 + 8 39, 2 + 6 32; fp32 16 units, 3000 + 6000 3 + 13 31.5, 4 + 12 27.5; 8 bits, 32 units, 4000 + 8000 1 + 7 35, 2 + 6 29.
struct WindowCost {
    double cache, cache_kb, text, text_kb;       // of a wave's tile of 32 rows, and of each KB of it
    double two, rate, begin, partial, split;     // more where a compute unit has two work-groups; MB a microsecond; a round of work-groups; a row's partial; of all rows at once
    int per_cu;                                  // work-groups that a compute unit has room for
};
constexpr WindowCost WINDOW_COST[4] = {          // bf16, fp32, 8 bits with rows of bf16 and of fp32
    {0.38, 0.066, 0.54, 0.086, 0.2, 6.7, 4.2, 0.00035, 0.029, 2},
    {0.25, 0.137, 0.52, 0.117, 0.13, 8.9, 9.3, 0.00033, 0.010, 1},
    {0.44, 0.071, 0.88, 0.049, 0.1, 6.6, 6.5, 0.00057, 0.022, 2},
    {1.58, 0.26, 2.4, 0.136, 0.17, 6.6, 7.1, 0.00028, 0.029, 2},
};
RowsPlan window_plan(const rk_ctx* ctx, const rk_layout* L, bool cache, int text_rows, bool q8)
{
    const bool f32 = L->dtype == RK_F32;
    const int64_t n_cu = ctx ? ctx->n_cu : 256, units = (int64_t)L->batch * L->n_kv_heads, slots = rows_slots(ctx, L, 1);
    const int nrb = (L->n_q_heads / L->n_kv_heads + 15) / 16;
    const int64_t groups = units * nrb;
    auto least = [](int64_t a, int64_t b) { return (int)(a < b ? a : b); };
    RowsPlan best;
    best.per = 16;
    best.nrb = nrb;
    if (!cache) {
        const int64_t wanted = text_rows < 1 ? 1 : ((int64_t)text_rows + 127) / 128;
        best.Sv = 0;
        best.Sr = least(least(n_cu / groups, wanted), slots);
        if (best.Sr < 1) best.Sr = 1;
        return best;
    }
    if (text_rows < 1 || (ctx && ctx->decode_splits > 0)) return rows_plan(ctx, L, 1, text_rows, false, q8, 16);
    const WindowCost& c = WINDOW_COST[(q8 ? 2 : 0) + (f32 ? 1 : 0)];
    const int r = keep_padded(L->keep), cached = L->max_seq_len < L->capacity ? L->max_seq_len : L->capacity;
    const double cache_kb = (q8 ? r + 132 : (r + D) * (f32 ? 4 : 2)) / 32.0, text_kb = 2 * D * (f32 ? 4 : 2) / 32.0;
    const int64_t tv = ((int64_t)cached + 31) / 32, tt = ((int64_t)text_rows + 31) / 32;
    const double kv = c.cache + c.cache_kb * cache_kb, kt = c.text + c.text_kb * text_kb, bytes = (double)units * (tv * cache_kb + tt * text_kb) * 1024 / (c.rate * 1e6);
    auto waves = [](int64_t tiles, int64_t splits) { return ((tiles + splits - 1) / splits + 3) / 4; };      // tiles of the longest wave
    double lowest = 1e300;
    for (const int sv : {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 32, 48}) {
        if (sv > 1 && (2 * sv > tv + 1 || sv >= slots)) break;
        const int64_t nv = waves(tv, sv), even = (int64_t)(kv * nv / kt);
        int before = 0;
        // as many for the text as take no longer than the cache's, or what is left of one work-group a compute unit, or of two
        for (const int64_t wish : {(tt + 4 * (even > 1 ? even : 1) - 1) / (4 * (even > 1 ? even : 1)), n_cu / groups - sv, 2 * n_cu / groups - sv}) {
            int sr = least(least(wish, (tt + 1) / 2), slots - sv);
            if (sr < 1) sr = 1;
            if (sr == before) continue;
            before = sr;
            const int64_t all = groups * (sv + sr), room = c.per_cu * n_cu;
            const double share = (double)all / n_cu, crowd = share < 1.0 ? 0.0 : share > 2.0 ? 1.0 : share - 1.0;
            const double v = kv * nv, t = kt * waves(tt, sr), longest = (v > t ? v : t) * (1.0 + c.two * crowd);
            const double cost = c.begin * ((all + room - 1) / room) + (longest > bytes ? longest : bytes) * (all > room ? (double)all / room : 1.0) +
                                c.partial * L->batch * L->n_q_heads * (sv + sr) + c.split * (sv + sr);
            if (cost < lowest) {
                lowest = cost;
                best.Sv = sv;
                best.Sr = sr;
            }
        }
    }
    return best;
}

// Prompts: rows of a block, blocks of a KV head, splits of what a block sees, whichever come out cheapest, in microseconds as measured. A work-group takes `each` for its
// beginning and end (`again` where others follow it), `edge` for a tile that is masked for some of its rows, and `step` for `tokens` of what it sees; no launch is shorter than its longest work-group (`alone` of a step while compute units are to spare), nor than all of them one
// after another on the compute units, where the last round is not full: that costs as much as a full one if they are equally long, and nothing if the short ones of a
// causal prompt fill it. Partials are written and read.
// us, bf16 with 32 / 256 rows a block: 8 units of 4 heads, 1 token on 1000 9.0 / 11.8, 40 on 4000 18.6 / 24.8, the same with a window of 512 11.7 / 17.9, 300 12.7 / 16.5, 700 28.1 /
// 25.9, 1000 42.6 / 32.1, 500 on 8000 175 / 77, 1500 on 2000 with a window of 512 71 / 32; 32 units of 7 heads, 20 on 500 11.9 / 20.3, 100 17.8 / 14.1, 40 on 4000 with
// a window of 512 24.1 / 27.8, 1000 283 / 90; 32 units of 1 head, 674 with a window of 55 18.4 / 27.5; 512 units of 4 heads, 4 on 500 28.6 / 45.4, 20 on 500 85 / 52.
// fp32 with 32 / 128 / 256 rows: 8 units of 4 heads, 8 on 4000 20.4 / 28.3 / 30.4, 40 on 1000 with a window of 512 16.6 / 21.9 / 24.2, 100 11.2 / 15.0 / 20.3, 300 23.6 / 27.0 / 29.8, 700
// 68 / 66 / 46, 500 on 8000 - / 525 / 339; 32 units of 7 heads, 100 29.8 / 22.4 / 25.6; 512 of 4, 4 on 500 62 / 131 / 153, 20 on 500 201 / 146 / 174; 32 units of 1 head, 1500 in 1, 2, 3, 4
// splits of 256 rows 190, 128, 140, 145, 2944 406, 416.  (Of 240 shapes drawn the plan's time was 1 % above the best of all rows and splits on average, 24 % at worst.)
// Where all work-groups run at once the longest is waited for, and a block takes a split for each so many tokens that it sees: less is begun, written and folded than with as many for all blocks.  us, all
// alike / by length: fp32 8 units of 4 heads, 300 in 5 splits 34 / 28, 1000 89 / 71, 2 units of 8 heads, 1000 58 / 47; bf16 8 units of 1 head, 3000 in 4 56 / 47.  Where they do not, the
// long ones have to come first, which they do with as many for all (fp32 4 units of 7 heads, 2944 in 2 363 / 385).
constexpr int PREFILL_SPLITS_MAX = 32, PREFILL_ROWS = 1024;
constexpr int64_t PREFILL_FAR = 1 << 24;         // elements between rows
struct PrefillPlan { int rows, blocks, S, tokens; };      // S: splits of a block; tokens not 0: one for each so many that it sees, up to S
// The first block of which a token may see more than `most` rows.
int prefill_cut(int rows, int64_t G, int n, int max_len, int64_t most)
{
    const int64_t token = most - ((int64_t)max_len - n);         // (the first to)
    return token <= 0 ? 0 : (int)(token * G / rows);
}
PrefillPlan prefill_plan(const rk_ctx* ctx, const rk_layout* L, int n, int max_len, int window, int sinks, int64_t stride_t = D)
{
    const int64_t units = (int64_t)L->batch * L->n_kv_heads, G = L->n_q_heads / L->n_kv_heads, n_cu = ctx ? ctx->n_cu : 256;
    PrefillPlan best{};
    double least = 1e300;
    auto look = [&](int rows, int tokens, int tile, double each, double again, double step, double alone, double edge) {
        const int64_t blocks = ((int64_t)n * G + rows - 1) / rows;
        // rows of the segment that a block sees: at most, and on average over the new tokens
        const double first = max_len > n ? (double)max_len - n + 1 : 1.0, last = max_len > 1 ? (double)max_len : 1.0;
        double most = last, seen = 0.5 * (first + last);
        const double bound = (double)window + sinks + rows / G + 1 + tile / 2;       // (a window begins inside a tile)
        if (window > 0 && bound < last) {
            most = bound;
            seen = bound <= first ? bound : (0.5 * (first + bound) * (bound - first) + bound * (last - bound)) / (last - first);
        }
        const double even = 2.0 * seen / most - 1.0;           // 1: all as long, 0: from nothing up
        const int64_t steps = (int64_t)((most + tokens - 1) / tokens), edges = (rows / G / tile + 1) * (window > 0 && bound < last ? 2 : 1);
        const double masked = edge * (edges < steps ? edges : steps);
        each += masked;
        again += masked;
        for (int S = 1; S <= PREFILL_SPLITS_MAX && S <= steps; ++S) {
            // (what the workspace holds)
            if (S > 1 && units * blocks * S * rows > PREFILL_ROWS * n_cu) break;
            const int64_t stretch = (steps + S - 1) / S;
            double parts = S;
            bool by_length = S > 1 && S <= PREFILL_CUTS + 1 && (S - 1) * stretch < steps && first <= (S - 1) * stretch * tokens;
            if (by_length) {
                int64_t all = blocks;
                for (int i = 1; i < S; ++i) all += blocks - prefill_cut(rows, G, n, max_len, i * stretch * tokens);
                by_length = units * all <= n_cu;
                if (by_length) parts = (double)all / blocks;
            }
            const double groups = (double)(units * blocks) * parts, share = groups / n_cu, full = (double)(int64_t)(share + 0.999);
            double rounds = share + (full - share) * (even > 0.0 ? even : 0.0);
            if (rounds < 1.0) rounds = 1.0;
            const double mean = seen / tokens / parts, longest = each + alone * stretch, all = (rounds > 1.0 ? again : each) * rounds + rounds * step * (mean > 1.0 ? mean : 1.0);
            const double merge = S == 1 ? 0.0 : 2.5 + 0.1 * S + (double)units * n * G * parts * 1040 / 4e6;
            const double cost = (longest > all ? longest : all) + merge;
            if (cost < least - 0.01) {
                least = cost;
                best = PrefillPlan{rows, (int)blocks, S, by_length ? (int)(stretch * tokens) : 0};
            }
        }
    };
    if (L->dtype == RK_F32) {
        look(32, 128, 32, 6.5, 12.0, 4.5, 4.5, 0.0);
        look(128, 32, 32, 5.0, 7.0, 4.5, 4.3, 0.0);
        look(256, 32, 32, 8.0, 11.0, 4.5, 4.2, 0.0);
    } else {
        if (stride_t < PREFILL_FAR) look(256, 64, 64, 7.0, 8.0, 1.55, 1.5, 2.0);       // (its lanes' addresses are 32 bits)
        look(32, 128, 32, 6.0, 6.5, 1.35, 1.35, 0.0);
    }
    return best;
}
// rows * splits of n tokens or fewer: at most PREFILL_SPLITS_MAX a row, and PREFILL_ROWS for each compute unit
size_t prefill_ws(const rk_ctx* ctx, const rk_layout* L, int n)
{
    const size_t rows = (size_t)L->batch * L->n_q_heads * n, most = (size_t)PREFILL_ROWS * (ctx ? ctx->n_cu : 256);
    const size_t slots = rows < most / PREFILL_SPLITS_MAX ? rows * PREFILL_SPLITS_MAX : most;
    return align_up(slots * (D + 2) * sizeof(float), 256) + 256;
}

// A launch has less than 2^32 threads along its first axis.
rk_status check_groups(rk_ctx* ctx, int64_t groups, int threads)
{
    if (groups <= (int64_t)UINT32_MAX / threads && groups <= INT32_MAX) return RK_OK;
    return fail(ctx, RK_ERR_UNSUPPORTED, "%lld work-groups of %d threads: more than a launch holds", (long long)groups, threads);
}
rk_status check_prefill_groups(rk_ctx* ctx, const rk_layout* L, const PrefillPlan& p)
{
    return check_groups(ctx, (int64_t)L->batch * L->n_kv_heads * p.blocks * p.S, L->dtype == RK_F32 && p.rows == 256 ? 512 : 256);
}
// of attn_rows, and of the fold behind it
rk_status check_rows_groups(rk_ctx* ctx, const rk_layout* L, const RowsPlan& p)
{
    const rk_status s = check_groups(ctx, ((int64_t)L->batch * L->n_kv_heads * (p.Sv + p.Sr) + 7) / 8 * 8 * p.nrb, 256);
    return s != RK_OK || p.Sv + p.Sr == 1 ? s : check_groups(ctx, ((int64_t)L->batch * L->n_q_heads + 7) / 8, 256);
}

rk_status check_window(rk_ctx* ctx, int32_t window, int32_t sinks)
{
    if (window < 0 || sinks < 0) return fail(ctx, RK_ERR_INVALID_ARG, "window %d, sinks %d: negative", window, sinks);
    return RK_OK;
}

rk_status check_heads(rk_ctx* ctx, const rk_heads* x, const char* name)
{
    if (!x || !x->data) return fail(ctx, RK_ERR_INVALID_ARG, "%s: NULL", name);
    if ((uintptr_t)x->data & 15) return fail(ctx, RK_ERR_INVALID_ARG, "%s: must be 16-byte aligned", name);
    if (x->stride_b < 0 || x->stride_h < 0 || x->stride_t < 0 || x->stride_b % 8 || x->stride_h % 8 || x->stride_t % 8)
        return fail(ctx, RK_ERR_INVALID_ARG, "%s: strides must be non-negative multiples of 8 elements", name);
    return RK_OK;
}
// Bytes from the first to the end of the last of B x H x n rows (strides are the caller's: more than 2^62 bytes are 2^62).
size_t heads_bytes(int64_t sb, int64_t sh, int64_t st, int B, int H, int n, size_t es)
{
    const __int128 bytes = ((__int128)(B - 1) * sb + (__int128)(H - 1) * sh + (__int128)(n - 1) * st + D) * es;
    return bytes < (__int128)1 << 62 ? (size_t)bytes : (size_t)1 << 62;
}

// Of a result: whether each row has elements of its own.  Sorted by their strides, each axis has to step over all that the axes below it cover (an
// axis of one does not step); heads of a projection's rows lie so.
bool rows_apart(const rk_heads* x, int B, int H, int n)
{
    const int64_t st[3] = {x->stride_b, x->stride_h, x->stride_t}, count[3] = {B, H, n};
    __int128 covered = D;
    bool done[3] = {B == 1, H == 1, n == 1};
    for (int k = 0; k < 3; ++k) {
        int at = -1;
        for (int i = 0; i < 3; ++i)
            if (!done[i] && (at < 0 || st[i] < st[at])) at = i;
        if (at < 0) return true;
        if (st[at] < covered) return false;
        covered += (__int128)(count[at] - 1) * st[at];
        done[at] = true;
    }
    return true;
}

rk_status check_result(rk_ctx* ctx, const rk_heads* x, const char* name, int B, int H, int n)
{
    const rk_status s = check_heads(ctx, x, name);
    if (s != RK_OK) return s;
    if (n > 0 && !rows_apart(x, B, H, n)) return fail(ctx, RK_ERR_INVALID_ARG, "%s: rows share elements", name);
    return RK_OK;
}

rk_status check_tokens(rk_ctx* ctx, const rk_layout* L, int32_t n)
{
    if (n < 0 || n > RK_MAX_TOKENS) return fail(ctx, RK_ERR_INVALID_ARG, "n_tokens %d outside 0..%d", n, RK_MAX_TOKENS);
    if ((int64_t)n * L->batch > INT32_MAX / L->n_q_heads) return fail(ctx, RK_ERR_UNSUPPORTED, "more than %d query rows", INT32_MAX);
    return RK_OK;
}
// (fewer than ROPE_TOKENS: a work-group a token)
rk_status check_rope_tokens(rk_ctx* ctx, const rk_layout* L, int32_t n)
{
    const rk_status s = check_tokens(ctx, L, n);
    return s != RK_OK ? s : check_groups(ctx, ((int64_t)n + ROPE_TOKENS - 1) / ROPE_TOKENS, 256);
}

rk_status check_rotary(rk_ctx* ctx, const rk_rotary* r)
{
    if (!r || !r->pos || !r->inv_freq) return fail(ctx, RK_ERR_INVALID_ARG, "rope: NULL, or NULL pos or inv_freq");
    if (r->n_axes < 1 || r->n_axes > RK_MAX_AXES) return fail(ctx, RK_ERR_INVALID_ARG, "rope: n_axes %d outside 1..%d", r->n_axes, RK_MAX_AXES);
    if (r->n_pairs < 1 || r->n_pairs > RK_MAX_PAIRS) return fail(ctx, RK_ERR_INVALID_ARG, "rope: n_pairs %d outside 1..%d", r->n_pairs, RK_MAX_PAIRS);
    if (r->pairing != RK_ROPE_HALVES && r->pairing != RK_ROPE_ADJACENT) return fail(ctx, RK_ERR_INVALID_ARG, "rope: unknown pairing %d", r->pairing);
    if (r->stride_a < 0 || r->stride_b < 0) return fail(ctx, RK_ERR_INVALID_ARG, "rope: negative strides of pos");
    for (int i = 0; i < r->n_pairs; ++i)
        if (r->axis[i] >= r->n_axes) return fail(ctx, RK_ERR_INVALID_ARG, "rope: axis %d of pair %d, of %d axes", r->axis[i], i, r->n_axes);
    return RK_OK;
}

RopeArgs rope_args(const rk_layout* L, const rk_rotary* r, int n, const int32_t* n_dev)
{
    RopeArgs a{};
    a.pos = r->pos; a.pos_sa = r->stride_a; a.pos_sb = r->stride_b; a.inv_freq = r->inv_freq;
    for (int i = 0; i < r->n_pairs; ++i) a.axes[i >> 5] |= (uint64_t)(r->axis[i] & 3) << (2 * (i & 31));
    a.n_axes = r->n_axes; a.n_pairs = r->n_pairs; a.pairing = r->pairing;
    a.B = L->batch; a.Hq = L->n_q_heads; a.Hkv = L->n_kv_heads; a.n = n; a.n_dev = n_dev;
    return a;
}

hipStream_t as_stream(void* s) { return (hipStream_t)s; }

// Makes `device` current for the duration of a call and puts the caller's device back
// afterwards: the library must not change the calling thread's current device.
struct DeviceGuard {
    int prev = -1;
    hipError_t status;
    explicit DeviceGuard(int device)
    {
        status = hipGetDevice(&prev);
        if (status == hipSuccess && prev != device) status = hipSetDevice(device);
        else if (status == hipSuccess) prev = -1;          // nothing to restore
    }
    ~DeviceGuard() { if (prev >= 0) (void)hipSetDevice(prev); }
    DeviceGuard(const DeviceGuard&) = delete;
    DeviceGuard& operator=(const DeviceGuard&) = delete;
};

}  // namespace

extern "C" {

const char* rk_status_str(rk_status s)
{
    switch (s) {
        case RK_OK: return "ok";
        case RK_ERR_INVALID_ARG: return "invalid argument";
        case RK_ERR_UNSUPPORTED: return "unsupported configuration";
        case RK_ERR_CAPACITY: return "cache capacity exceeded";
        case RK_ERR_WORKSPACE: return "workspace missing or too small";
        case RK_ERR_HIP: return "HIP error";
        case RK_ERR_NO_DEVICE: return "context has no device";
    }
    return "unknown status";
}

rk_status rk_create(rk_ctx** out, int device)
{
    if (!out) return RK_ERR_INVALID_ARG;
    *out = nullptr;
    rk_ctx* c = new (std::nothrow) rk_ctx();
    if (!c) return RK_ERR_INVALID_ARG;
    memset(c, 0, sizeof(*c));
    c->device = device;
    c->n_cu = 256;
    c->fuse_merge = 1;
    if (device != RK_DEVICE_NONE) {
        if (device < 0) { delete c; return RK_ERR_INVALID_ARG; }
        hipDeviceProp_t prop;
        hipError_t e = hipGetDeviceProperties(&prop, device);
        if (e != hipSuccess) { delete c; return RK_ERR_HIP; }
        c->n_cu = prop.multiProcessorCount > 0 ? prop.multiProcessorCount : 256;
        const size_t tb = (size_t)(APP_TICKETS + DEC_COUNTERS) * sizeof(int32_t);
        DeviceGuard dev(device);
        if (dev.status != hipSuccess || hipMalloc((void**)&c->tickets, tb) != hipSuccess) {
            delete c;
            return RK_ERR_HIP;
        }
        if (hipMemset(c->tickets, 0, tb) != hipSuccess || hipDeviceSynchronize() != hipSuccess) {
            (void)hipFree(c->tickets);
            delete c;
            return RK_ERR_HIP;
        }
        // the folded merge needs all work-groups of a unit behind one L2: check how this device deals them
        bool same_xcd = false;
        if (probe_xcd_deal(c->tickets, &same_xcd) != hipSuccess) {
            (void)hipFree(c->tickets);
            delete c;
            return RK_ERR_HIP;
        }
        c->xcd_deal_ok = same_xcd ? 1 : 0;
        // this device's copy of the static scratch array (each GPU has its own, at its own address)
        if (hipGetSymbolAddress(&c->static_scratch, HIP_SYMBOL(scratch)) != hipSuccess || !c->static_scratch) {
            (void)hipFree(c->tickets);
            delete c;
            return RK_ERR_HIP;
        }
    }
    *out = c;
    return RK_OK;
}

rk_status rk_destroy(rk_ctx* ctx)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    if (ctx->tickets) {
        DeviceGuard dev(ctx->device);
        (void)hipFree(ctx->tickets);
    }
    delete ctx;
    return RK_OK;
}

const char* rk_last_error(const rk_ctx* ctx) { return ctx ? ctx->err : "context is NULL"; }

rk_status rk_set_option(rk_ctx* ctx, int32_t key, int64_t value)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    switch (key) {
        case RK_OPT_FORCE_GENERIC: ctx->force_generic = value != 0; return RK_OK;
        case RK_OPT_FUSE_MERGE: ctx->fuse_merge = value != 0; return RK_OK;
        case RK_OPT_DECODE_SPLITS:
            if (value < 0 || value > 4096) return fail(ctx, RK_ERR_INVALID_ARG, "decode splits %lld outside 0..4096", (long long)value);
            ctx->decode_splits = (int)value;
            return RK_OK;
        default: return fail(ctx, RK_ERR_INVALID_ARG, "unknown option %d", key);
    }
}

rk_status rk_validate_layout(const rk_layout* L) { return check_layout(nullptr, L); }

size_t rk_fit_workspace_size(const rk_layout* L, int32_t max_tokens)
{
    if (check_layout(nullptr, L) != RK_OK || max_tokens < 0 || max_tokens > RK_MAX_TOKENS) return 0;
    return fit_ws(L, max_tokens).total;
}

size_t rk_decode_workspace_size(const rk_ctx* ctx, const rk_layout* L)
{
    if (check_layout(nullptr, L) != RK_OK) return 0;
    return decode_plan(ctx, L).bytes;
}

rk_status rk_decode_plan(const rk_ctx* ctx, const rk_layout* L, int32_t* n_splits, int32_t* tokens_per_split)
{
    rk_status s = check_layout(nullptr, L);
    if (s != RK_OK) return s;
    if (!n_splits || !tokens_per_split) return RK_ERR_INVALID_ARG;
    const DecodePlan p = decode_plan(ctx, L);
    *n_splits = p.S;
    *tokens_per_split = 128 * ((p.tiles + p.S - 1) / p.S);      // the largest split
    return RK_OK;
}

rk_status rk_cache_bytes(const rk_layout* L, size_t* k_packed_bytes, size_t* v_cache_bytes)
{
    rk_status s = check_layout(nullptr, L);
    if (s != RK_OK) return s;
    const size_t slabs = (size_t)L->batch * L->n_kv_heads * slab_tokens(L->capacity);       // slabs are spaced, see slab_tokens()
    if (k_packed_bytes) *k_packed_bytes = slabs * keep_padded(L->keep) * elem_size(L->dtype);
    if (v_cache_bytes) *v_cache_bytes = slabs * D * elem_size(L->dtype);
    return RK_OK;
}

rk_status rk_unpack_cache(rk_ctx* ctx, const rk_layout* L, const void* k_packed, const void* v_cache,
                          void* k_rows, void* v_rows, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if ((k_rows && !k_packed) || (v_rows && !v_cache) || (!k_rows && !v_rows))
        return fail(ctx, RK_ERR_INVALID_ARG, "unpack: nothing to do or source missing");
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_unpack(L->dtype, L->batch * L->n_kv_heads, L->capacity, L->keep, k_packed, v_cache, k_rows, v_rows,
                      as_stream(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "unpack launch");
    return RK_OK;
}

rk_status rk_stream_read(rk_ctx* ctx, const void* src, size_t bytes, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    if (!src || ((uintptr_t)src & 15) || bytes == 0 || (bytes & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "stream_read: src must be non-NULL and 16-byte aligned, bytes a positive multiple of 16");
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_stream_read(src, bytes, ctx->n_cu, nullptr, as_stream(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "stream_read launch");
    return RK_OK;
}

rk_status rk_fit_rotation(rk_ctx* ctx, const rk_layout* L, const rk_rows* keys, const float* sigma,
                          uint32_t flags, const rk_fit_out* out, void* workspace, size_t workspace_bytes,
                          void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    s = check_rows(ctx, L, keys, "keys");
    if (s != RK_OK) return s;
    if (!out || !out->R || !out->eigvals || !out->mask || !out->keep_idx || !out->R_r || !out->mu || !out->delta_mu)
        return fail(ctx, RK_ERR_INVALID_ARG, "fit outputs: a required pointer is NULL");
    if (flags & ~(uint32_t)RK_FIT_CENTER) return fail(ctx, RK_ERR_INVALID_ARG, "unknown fit flags 0x%x", flags);
    const FitWs w = fit_ws(L, keys->n_tokens);
    if (!workspace || workspace_bytes < w.total || ((uintptr_t)workspace & 255))
        return fail(ctx, RK_ERR_WORKSPACE, "fit workspace: need %zu bytes, 256-byte aligned", w.total);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");

    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    const int B = L->batch, Hkv = L->n_kv_heads, U = B * Hkv;
    const bool mfma = !ctx->force_generic;
    const int ct = cov_chunk_tokens(L->dtype, mfma, U, keys->n_tokens, ctx->n_cu);
    int nc = (keys->n_tokens + ct - 1) / ct;        // never more than the workspace was sized for
    if (nc < 1) nc = 1;
    char* ws = (char*)workspace;
    float* part_S = (float*)(ws + w.part_S);
    float* part_sum = (float*)(ws + w.part_sum);
    float* cov = out->cov ? out->cov : (float*)(ws + w.cov);
    const RowsDev rows = to_dev(keys);
    hipStream_t st = as_stream(stream);
    e = launch_cov_partial(L->dtype, mfma, rows, B, Hkv, nc, ct, part_S, part_sum, st);
    if (e != hipSuccess) return hip_fail(ctx, e, "covariance launch");
    e = launch_cov_finalize(L->dtype, mfma, rows, B, Hkv, nc, ct, (flags & RK_FIT_CENTER) != 0, part_S, part_sum, cov, out->mu, ctx->n_cu, st);
    if (e != hipSuccess) return hip_fail(ctx, e, "covariance reduction launch");
    e = launch_eig(ctx->force_generic != 0, U, cov, sigma, out->mu, L->keep, out->R, out->eigvals, out->mask, out->keep_idx, out->R_r,
                   out->delta_mu, out->sweeps, ws + w.part_S, (int32_t*)(ws + w.status), st);
    if (e != hipSuccess) return hip_fail(ctx, e, "eigensolver launch");
    return RK_OK;
}

rk_status rk_query_sigma(rk_ctx* ctx, const rk_layout* L, const void* q_window, int64_t stride_b, int64_t stride_h,
                         int64_t stride_w, int32_t window, float* sigma, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!q_window || !sigma) return fail(ctx, RK_ERR_INVALID_ARG, "query_sigma: NULL pointer");
    if (window < 1) return fail(ctx, RK_ERR_INVALID_ARG, "query_sigma: window must be >= 1");
    if (stride_b < 0 || stride_h < 0 || stride_w < D)
        return fail(ctx, RK_ERR_INVALID_ARG, "query_sigma: strides must be non-negative, stride_w >= %d", D);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_sigma_window(L->dtype, q_window, stride_b, stride_h, stride_w, L->batch, L->n_q_heads, L->n_kv_heads,
                            window, sigma, as_stream(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "query_sigma launch");
    return RK_OK;
}

rk_status rk_fit_subspace(rk_ctx* ctx, const rk_layout* L, const rk_rows* keys, const float* sigma, uint32_t flags,
                          const rk_subspace* solver, float* R_r, float* mu, float* delta_mu, float* cov_out,
                          int32_t* status, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    s = check_rows(ctx, L, keys, "keys");
    if (s != RK_OK) return s;
    if (!solver || !solver->v0) return fail(ctx, RK_ERR_INVALID_ARG, "fit_subspace: solver or its start basis is NULL");
    if (solver->iterations < 1 || !(solver->ridge >= 0.0))
        return fail(ctx, RK_ERR_INVALID_ARG, "fit_subspace: iterations must be >= 1 and ridge >= 0");
    if (!R_r || !mu || !delta_mu) return fail(ctx, RK_ERR_INVALID_ARG, "fit_subspace: a required output is NULL");
    if (flags & ~(uint32_t)RK_FIT_CENTER) return fail(ctx, RK_ERR_INVALID_ARG, "unknown fit flags 0x%x", flags);
    if (L->keep > subspace_max_keep())
        return fail(ctx, RK_ERR_UNSUPPORTED, "fit_subspace: keep %d exceeds %d; use rk_fit_rotation", L->keep,
                    subspace_max_keep());
    const FitWs w = fit_ws(L, keys->n_tokens);
    if (!workspace || workspace_bytes < w.total || ((uintptr_t)workspace & 255))
        return fail(ctx, RK_ERR_WORKSPACE, "fit workspace: need %zu bytes, 256-byte aligned", w.total);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");

    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    const int B = L->batch, Hkv = L->n_kv_heads, U = B * Hkv;
    const bool mfma = !ctx->force_generic;
    const int ct = cov_chunk_tokens(L->dtype, mfma, U, keys->n_tokens, ctx->n_cu);
    int nc = (keys->n_tokens + ct - 1) / ct;
    if (nc < 1) nc = 1;
    char* ws = (char*)workspace;
    float* part_S = (float*)(ws + w.part_S);
    float* part_sum = (float*)(ws + w.part_sum);
    float* cov = cov_out ? cov_out : (float*)(ws + w.cov);
    const RowsDev rows = to_dev(keys);
    hipStream_t st = as_stream(stream);
    e = launch_cov_partial(L->dtype, mfma, rows, B, Hkv, nc, ct, part_S, part_sum, st);
    if (e != hipSuccess) return hip_fail(ctx, e, "covariance launch");
    e = launch_cov_finalize(L->dtype, mfma, rows, B, Hkv, nc, ct, (flags & RK_FIT_CENTER) != 0, part_S, part_sum, cov, mu, ctx->n_cu, st);
    if (e != hipSuccess) return hip_fail(ctx, e, "covariance reduction launch");
    e = launch_subspace(U, cov, sigma, mu, solver->v0, L->keep, solver->iterations, solver->ridge, R_r, delta_mu,
                        status, st);
    if (e != hipSuccess) return hip_fail(ctx, e, "subspace iteration launch");
    return RK_OK;
}

rk_status rk_gather_rotation(rk_ctx* ctx, const rk_layout* L, const float* R, const int32_t* keep_idx,
                             float* R_r, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!R || !keep_idx || !R_r) return fail(ctx, RK_ERR_INVALID_ARG, "gather_rotation: NULL pointer");
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_gather_rotation(L->batch * L->n_kv_heads, L->keep, R, keep_idx, R_r, as_stream(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "gather launch");
    return RK_OK;
}

rk_status rk_compress(rk_ctx* ctx, const rk_layout* L, const rk_rows* keys, const float* R_r, void* k_packed,
                      const rk_rows* values, void* v_cache, int32_t* seq_len_out, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    s = check_rows(ctx, L, keys, "keys");
    if (s != RK_OK) return s;
    if (!R_r || !k_packed) return fail(ctx, RK_ERR_INVALID_ARG, "compress: R_r or k_packed is NULL");
    if ((uintptr_t)k_packed & 15) return fail(ctx, RK_ERR_INVALID_ARG, "compress: k_packed must be 16-byte aligned");
    if (values) {
        s = check_rows(ctx, L, values, "values");
        if (s != RK_OK) return s;
        if (!v_cache || ((uintptr_t)v_cache & 15))
            return fail(ctx, RK_ERR_INVALID_ARG, "compress: values given but v_cache is NULL or misaligned");
        if (values->n_tokens != keys->n_tokens || values->tok_idx != keys->tok_idx ||
            values->tok_off != keys->tok_off || values->n_tokens_dev != keys->n_tokens_dev)
            return fail(ctx, RK_ERR_INVALID_ARG, "compress: values must use the same row selection as keys");
    }
    if (keys->n_tokens > L->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "compress: %d rows exceed capacity %d", keys->n_tokens, L->capacity);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");

    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    hipStream_t st = as_stream(stream);
    RowsDev vals;
    bool join = false;
    if (values) {
        vals = to_dev(values);
        // One launch for Keys and Values, except where the Value cache lies over the Keys or R_r, which must have been read by then, and
        // through token lists, for which there is no such kernel.  (Every row's address comes from a load there, and the few work-groups that fit
        // beside the rotation's registers do not hide two round trips where they are many: a prefill of 4 x 32 heads, 4128 listed rows, r = 32, took 187 us
        // instead of 178; that is beyond the line at which bf16 is joined at all.  Within it lists would gain as well: two launches / one, us, 1 x 8 x 2410
        // listed rows, r = 64, 11.7 / 9.4; 1 x 32 x 3000 18.6 / 16.8; 4 x 32 x 1000 ragged 20.8 / 21.4, r = 128 27.0 / 25.4.)
        const size_t es = elem_size(L->dtype), units = (size_t)L->batch * L->n_kv_heads;
        const size_t kb = (size_t)((L->batch - 1) * keys->stride_b + (L->n_kv_heads - 1) * keys->stride_h +
                                   (int64_t)(keys->n_tokens > 0 ? keys->n_tokens - 1 : 0) * keys->stride_t + D) * es;
        const size_t vb = units * slab_tokens(L->capacity) * D * es;
        join = !keys->tok_idx && !ranges_meet(v_cache, vb, keys->data, kb) && !ranges_meet(v_cache, vb, R_r, units * D * L->keep * sizeof(float));
    }
    e = launch_compress(L->dtype, !ctx->force_generic, to_dev(keys), L->batch, L->n_kv_heads, L->capacity, L->keep,
                        R_r, k_packed, seq_len_out, values ? &vals : nullptr, v_cache, join, ctx->n_cu, st);
    return e == hipSuccess ? RK_OK : hip_fail(ctx, e, "compress launch");
}

rk_status rk_append(rk_ctx* ctx, const rk_layout* L, const void* k_new, const void* v_new, const float* R_r,
                    void* k_packed, void* v_cache, int32_t* seq_len, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!k_new || !v_new || !R_r || !k_packed || !v_cache || !seq_len)
        return fail(ctx, RK_ERR_INVALID_ARG, "append: NULL pointer");
    if (L->max_seq_len + 1 > L->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "append: %d + 1 rows exceed capacity %d", L->max_seq_len, L->capacity);
    if (L->batch > APP_TICKETS) return fail(ctx, RK_ERR_UNSUPPORTED, "append: batch too large");
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_append(L->dtype, L->batch, L->n_kv_heads, L->capacity, L->keep, k_new, v_new, R_r, k_packed,
                      v_cache, seq_len, ctx->tickets, as_stream(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "append launch");
    return RK_OK;
}

// tk_new / tv_new non-null: one row per sequence joins the text segment inside the same launches
static rk_status decode_common(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_packed,
                               const void* v_cache, const float* R_r, const float* delta_mu, const rk_text* text,
                               const void* tk_new, const void* tv_new, float scale, void* out, void* workspace,
                               size_t workspace_bytes, void* stream, bool use_static = false)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!q || !k_packed || !v_cache || !R_r || !out || !L->seq_len)
        return fail(ctx, RK_ERR_INVALID_ARG, "decode: NULL pointer (q, k_packed, v_cache, R_r, out, seq_len)");
    if (((uintptr_t)k_packed & 15) || ((uintptr_t)v_cache & 15) || ((uintptr_t)q & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "decode: q and the caches must be 16-byte aligned");
    if (L->max_seq_len > L->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "decode: max_seq_len %d exceeds capacity %d", L->max_seq_len, L->capacity);
    TextDev td{};
    TextAppendDev ta{};
    if (text) {
        s = check_text(ctx, text, tk_new != nullptr);
        if (s != RK_OK) return s;
        td = TextDev{text->k, text->v, text->stride_b, text->stride_h, text->stride_t, text->len, text->max_len};
        if (tk_new) {
            if (!tv_new || ((uintptr_t)tk_new & 15) || ((uintptr_t)tv_new & 15))
                return fail(ctx, RK_ERR_INVALID_ARG, "append_text_decode: k_new, v_new must be non-NULL, 16-byte aligned");
            if (text->max_len + 1 > text->capacity)
                return fail(ctx, RK_ERR_CAPACITY, "append_text_decode: %d + 1 rows exceed capacity %d", text->max_len,
                            text->capacity);
            td.max_len = text->max_len + 1;
            ta = TextAppendDev{text->k, text->v, tk_new, tv_new, text->stride_b, text->stride_h, text->stride_t,
                               text->len, text->capacity};
        }
    }
    const DecodePlan p = decode_plan(ctx, L, text ? td.max_len : 0);
    const size_t need = p.bytes;
    if (use_static) {
        if (need > (size_t)RK_STATIC_SCRATCH_BYTES)
            return fail(ctx, RK_ERR_WORKSPACE, "decode (static scratch): this shape needs %zu bytes of partials, the "
                        "built-in scratch holds %zu; use rk_decode_attn with a workspace", need,
                        (size_t)RK_STATIC_SCRATCH_BYTES);
        if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
        workspace = ctx->static_scratch;            // the device address taken at rk_create, never the symbol
    } else if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))
        return fail(ctx, RK_ERR_WORKSPACE, "decode workspace: need %zu bytes, 16-byte aligned", need);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");

    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    const int S = p.S;
    const int St = text && L->dtype == RK_BF16 && use_mfma_decode(ctx, L) ? text_splits(ctx, L, S, td.max_len) : 0;
    const float sc = scale > 0.f ? scale : 1.0f / sqrtf((float)L->head_dim);
    e = launch_decode(L->dtype, use_mfma_decode(ctx, L), L->batch, L->n_q_heads, L->n_kv_heads, L->capacity,
                      L->keep, S + St, S, p.tiles, q, k_packed, v_cache, R_r, delta_mu, L->seq_len, text ? &td : nullptr, nullptr,
                      tk_new ? &ta : nullptr, sc, out, (float*)workspace,
                      ctx->fuse_merge && ctx->xcd_deal_ok ? ctx->tickets + APP_TICKETS : nullptr, DEC_COUNTERS,
                      L->batch <= APP_TICKETS ? ctx->tickets : nullptr, ctx->n_cu, as_stream(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "decode launch");
    return RK_OK;
}

rk_status rk_decode_attn(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_packed,
                         const void* v_cache, const float* R_r, const float* delta_mu, float scale, void* out,
                         void* workspace, size_t workspace_bytes, void* stream)
{
    return decode_common(ctx, L, q, k_packed, v_cache, R_r, delta_mu, nullptr, nullptr, nullptr, scale, out,
                         workspace, workspace_bytes, stream);
}

rk_status rk_decode_attn_static(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_packed,
                                const void* v_cache, const float* R_r, const float* delta_mu, float scale,
                                void* out, void* stream)
{
    return decode_common(ctx, L, q, k_packed, v_cache, R_r, delta_mu, nullptr, nullptr, nullptr, scale, out,
                         nullptr, 0, stream, true);
}

rk_status rk_decode_attn_dual(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_packed,
                              const void* v_cache, const float* R_r, const float* delta_mu, const rk_text* text,
                              float scale, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    if (!text) return fail(ctx, RK_ERR_INVALID_ARG, "decode (dual): text is NULL");
    return decode_common(ctx, L, q, k_packed, v_cache, R_r, delta_mu, text, nullptr, nullptr, scale, out, workspace,
                         workspace_bytes, stream);
}

rk_status rk_append_text_decode_attn_dual(rk_ctx* ctx, const rk_layout* L, const void* k_new, const void* v_new,
                                          const void* q, const void* k_packed, const void* v_cache,
                                          const float* R_r, const float* delta_mu, const rk_text* text, float scale,
                                          void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    if (!text) return fail(ctx, RK_ERR_INVALID_ARG, "append_text_decode: text is NULL");
    if (!k_new || !v_new) return fail(ctx, RK_ERR_INVALID_ARG, "append_text_decode: NULL pointer (k_new, v_new)");
    return decode_common(ctx, L, q, k_packed, v_cache, R_r, delta_mu, text, k_new, v_new, scale, out, workspace,
                         workspace_bytes, stream);
}

rk_status rk_append_decode_attn(rk_ctx* ctx, const rk_layout* L, const void* k_new, const void* v_new, const void* q,
                                const float* R_r, const float* delta_mu, void* k_packed, void* v_cache,
                                int32_t* seq_len, float scale, void* out, void* workspace, size_t workspace_bytes,
                                void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!k_new || !v_new || !q || !R_r || !k_packed || !v_cache || !seq_len || !out)
        return fail(ctx, RK_ERR_INVALID_ARG, "append_decode: NULL pointer");
    if (((uintptr_t)k_packed & 15) || ((uintptr_t)v_cache & 15) || ((uintptr_t)k_new & 15) || ((uintptr_t)v_new & 15) ||
        ((uintptr_t)q & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "append_decode: q, k_new, v_new and the caches must be 16-byte aligned");
    if (L->max_seq_len + 1 > L->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "append_decode: %d + 1 rows exceed capacity %d", L->max_seq_len,
                    L->capacity);
    if (L->batch > APP_TICKETS) return fail(ctx, RK_ERR_UNSUPPORTED, "append_decode: batch too large");
    // everything below is planned for the length after the append
    rk_layout La = *L;
    La.max_seq_len = L->max_seq_len + 1;
    La.seq_len = seq_len;
    const DecodePlan p = decode_plan(ctx, &La);
    const size_t need = p.bytes;
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))
        return fail(ctx, RK_ERR_WORKSPACE, "append_decode workspace: need %zu bytes, 16-byte aligned", need);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");

    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    hipStream_t st = as_stream(stream);
    const float sc = scale > 0.f ? scale : 1.0f / sqrtf((float)L->head_dim);
    const bool mfma = use_mfma_decode(ctx, L);
    const AppendDev app{k_new, v_new, seq_len};
    const bool fused = decode_append_fusable(L->dtype, mfma, L->n_q_heads, L->n_kv_heads, L->keep);
    if (!fused) {
        // no free matrix-core column (G >= 16) or the plain kernels: the two steps run
        // as the launches of rk_append and rk_decode_attn
        e = launch_append(L->dtype, L->batch, L->n_kv_heads, L->capacity, L->keep, k_new, v_new, R_r, k_packed,
                          v_cache, seq_len, ctx->tickets, st);
        if (e != hipSuccess) return hip_fail(ctx, e, "append launch");
    }
    e = launch_decode(L->dtype, mfma, L->batch, L->n_q_heads, L->n_kv_heads, L->capacity, L->keep, p.S, p.S, p.tiles, q,
                      k_packed, v_cache, R_r, delta_mu, seq_len, nullptr, fused ? &app : nullptr, nullptr, sc, out,
                      (float*)workspace, ctx->fuse_merge && ctx->xcd_deal_ok ? ctx->tickets + APP_TICKETS : nullptr,
                      DEC_COUNTERS, ctx->tickets, ctx->n_cu, st);
    if (e != hipSuccess) return hip_fail(ctx, e, "decode launch");
    return RK_OK;
}

rk_status rk_append_text(rk_ctx* ctx, const rk_layout* L, const rk_text* text, const void* k_new,
                         const void* v_new, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!text) return fail(ctx, RK_ERR_INVALID_ARG, "append_text: text is NULL");
    s = check_text(ctx, text, true);
    if (s != RK_OK) return s;
    if (!k_new || !v_new) return fail(ctx, RK_ERR_INVALID_ARG, "append_text: NULL pointer (k_new, v_new)");
    if (text->max_len + 1 > text->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "append_text: %d + 1 rows exceed capacity %d", text->max_len,
                    text->capacity);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_append_text(L->dtype, L->batch, L->n_kv_heads, text->capacity, k_new, v_new, text->k, text->v,
                           text->stride_b, text->stride_h, text->stride_t, text->len, as_stream(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "append_text launch");
    return RK_OK;
}

rk_status rk_cache_bytes_quant(const rk_layout* L, size_t* k_q8_bytes, size_t* v_q8_bytes)
{
    rk_status s = check_layout(nullptr, L);
    if (s != RK_OK) return s;
    const size_t slabs = (size_t)L->batch * L->n_kv_heads * slab_tokens(L->capacity);
    if (k_q8_bytes) *k_q8_bytes = slabs / 32 * q8_kblock(keep_padded(L->keep));
    if (v_q8_bytes) *v_q8_bytes = slabs * D;
    return RK_OK;
}

rk_status rk_compress_quant(rk_ctx* ctx, const rk_layout* L, const rk_rows* keys, const float* R_r, void* k_q8,
                         const rk_rows* values, void* v_q8, int32_t* seq_len_out, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    s = check_rows(ctx, L, keys, "keys");
    if (s != RK_OK) return s;
    s = check_rows(ctx, L, values, "values");
    if (s != RK_OK) return s;
    if (!R_r || !k_q8 || !v_q8) return fail(ctx, RK_ERR_INVALID_ARG, "compress_quant: R_r, k_q8 or v_q8 is NULL");
    if (((uintptr_t)k_q8 & 15) || ((uintptr_t)v_q8 & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "compress_quant: the caches must be 16-byte aligned");
    if (values->n_tokens != keys->n_tokens || values->tok_idx != keys->tok_idx || values->tok_off != keys->tok_off ||
        values->n_tokens_dev != keys->n_tokens_dev)
        return fail(ctx, RK_ERR_INVALID_ARG, "compress_quant: values must use the same row selection as keys");
    if (keys->n_tokens > L->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "compress_quant: %d rows exceed capacity %d", keys->n_tokens, L->capacity);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_compress_q8(L->dtype, to_dev(keys), to_dev(values), L->batch, L->n_kv_heads, L->capacity, L->keep, R_r, k_q8, v_q8,
                           seq_len_out, ctx->n_cu, as_stream(stream));
    return e == hipSuccess ? RK_OK : hip_fail(ctx, e, "compress_quant launch");
}

rk_status rk_append_quant(rk_ctx* ctx, const rk_layout* L, const void* k_new, const void* v_new, const float* R_r, void* k_q8,
                       void* v_q8, int32_t* seq_len_out, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!k_new || !v_new || !R_r || !k_q8 || !v_q8 || !L->seq_len || !seq_len_out)
        return fail(ctx, RK_ERR_INVALID_ARG, "append_quant: NULL pointer");
    if (((uintptr_t)k_q8 & 15) || ((uintptr_t)v_q8 & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "append_quant: the caches must be 16-byte aligned");
    if (L->max_seq_len + 1 > L->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "append_quant: %d + 1 rows exceed capacity %d", L->max_seq_len, L->capacity);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_append_q8(L->dtype, L->batch, L->n_kv_heads, L->capacity, L->keep, k_new, v_new, R_r, k_q8, v_q8, L->seq_len,
                         seq_len_out, ctx->tickets, as_stream(stream));
    return e == hipSuccess ? RK_OK : hip_fail(ctx, e, "append_quant launch");
}

rk_status rk_unpack_cache_quant(rk_ctx* ctx, const rk_layout* L, const void* k_q8, const void* v_q8, void* k_rows, void* v_rows,
                             void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!k_q8 || (v_rows && !v_q8) || (!k_rows && !v_rows))       // (the steps of the Values lie beside the Keys')
        return fail(ctx, RK_ERR_INVALID_ARG, "unpack_quant: nothing to do or source missing");
    if (((uintptr_t)k_q8 & 15) || ((uintptr_t)v_q8 & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "unpack_quant: the caches must be 16-byte aligned");
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    e = launch_unpack_q8(L->dtype, L->batch, L->n_kv_heads, L->capacity, L->keep, k_q8, v_q8, L->seq_len, k_rows, v_rows,
                         as_stream(stream));
    return e == hipSuccess ? RK_OK : hip_fail(ctx, e, "unpack_quant launch");
}

size_t rk_tree_workspace_size(const rk_ctx* ctx, const rk_layout* L, int32_t n_tokens)
{
    if (check_layout(nullptr, L) != RK_OK || n_tokens < 1 || n_tokens > RK_MAX_DRAFTS) return 0;
    return rows_ws(ctx, L, n_tokens);
}

rk_status rk_tree_plan(const rk_ctx* ctx, const rk_layout* L, int32_t n_tokens, int32_t text_rows, int32_t quant, int32_t* rows_per_work_group,
                       int32_t* n_splits, int32_t* n_text_splits)
{
    const rk_status s = check_layout(nullptr, L);
    if (s != RK_OK) return s;
    if (n_tokens < 0 || n_tokens > RK_MAX_DRAFTS || text_rows < 0 || !rows_per_work_group || !n_splits || !n_text_splits) return RK_ERR_INVALID_ARG;
    const RowsPlan p = rows_plan(ctx, L, n_tokens ? n_tokens : 1, text_rows, n_tokens > 0, quant != 0);
    *rows_per_work_group = p.per;
    *n_splits = p.Sv;
    *n_text_splits = p.Sr;
    return RK_OK;
}

static rk_status check_drafts(rk_ctx* ctx, const rk_drafts* d)
{
    if (!d || !d->k || !d->v) return fail(ctx, RK_ERR_INVALID_ARG, "drafts: NULL, or NULL k or v");
    if (((uintptr_t)d->k & 15) || ((uintptr_t)d->v & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "drafts: k and v must be 16-byte aligned");
    if (d->n_tokens < 1 || d->n_tokens > RK_MAX_DRAFTS)
        return fail(ctx, RK_ERR_INVALID_ARG, "drafts: n_tokens %d outside 1..%d", d->n_tokens, RK_MAX_DRAFTS);
    if (d->stride_b < 0 || d->stride_h < 0 || d->stride_t < D || (d->stride_b % 8) || (d->stride_h % 8) || (d->stride_t % 8))
        return fail(ctx, RK_ERR_INVALID_ARG, "drafts: strides must be non-negative multiples of 8 elements, stride_t >= %d", D);
    if ((uintptr_t)d->mask & 7) return fail(ctx, RK_ERR_INVALID_ARG, "drafts: mask must be 8-byte aligned");
    return RK_OK;
}

static rk_status rows_common(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_cache, const void* v_cache,
                             const float* R_r, const float* delta_mu, const rk_text* text, const rk_drafts* drafts, bool q8,
                             float scale, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!q || !k_cache || !v_cache || !R_r || !out || !L->seq_len)
        return fail(ctx, RK_ERR_INVALID_ARG, "attention: NULL pointer (q, caches, R_r, out, seq_len)");
    if (((uintptr_t)k_cache & 15) || ((uintptr_t)v_cache & 15) || ((uintptr_t)q & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "attention: q and the caches must be 16-byte aligned");
    if (L->max_seq_len > L->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "attention: max_seq_len %d exceeds capacity %d", L->max_seq_len, L->capacity);
    if (text && (s = check_text(ctx, text, false)) != RK_OK) return s;
    const int T = drafts ? drafts->n_tokens : 1;
    if ((int64_t)L->batch * T * L->n_q_heads > INT32_MAX)
        return fail(ctx, RK_ERR_UNSUPPORTED, "attention: more than %d query rows", INT32_MAX);
    const size_t need = rows_ws(ctx, L, T);
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))
        return fail(ctx, RK_ERR_WORKSPACE, "attention workspace: need %zu bytes, 16-byte aligned", need);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");

    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    const RowsPlan p = rows_plan(ctx, L, T, text ? text->max_len : 0, drafts != nullptr, q8);
    RowsArgs a{};
    a.q = q; a.Kc = k_cache; a.Vc = v_cache; a.Rr = R_r; a.dmu = delta_mu; a.seq_len = L->seq_len; a.out = out;
    a.B = L->batch; a.T = T; a.Hq = L->n_q_heads; a.Hkv = L->n_kv_heads; a.G = a.Hq / a.Hkv;
    a.cap = L->capacity; a.r = L->keep; a.rp = keep_padded(L->keep);
    a.Sv = p.Sv; a.Sr = p.Sr; a.nrb = p.nrb;
    const float sc = scale > 0.f ? scale : 1.0f / sqrtf((float)L->head_dim);
    a.scale_log2 = sc * 1.44269504088896340736f;
    if (text) {
        a.text_k = text->k; a.text_v = text->v; a.text_len = text->len; a.text_max = text->max_len;
        a.text_sb = text->stride_b; a.text_sh = text->stride_h; a.text_st = text->stride_t;
    }
    if (drafts) {
        a.draft_k = drafts->k; a.draft_v = drafts->v; a.n_drafts = drafts->n_tokens_dev; a.mask = drafts->mask;
        a.draft_sb = drafts->stride_b; a.draft_sh = drafts->stride_h; a.draft_st = drafts->stride_t;
    }
    const size_t slots = (size_t)a.B * T * a.Hq * (p.Sv + p.Sr);
    a.ws_acc = (float*)align_up((uintptr_t)workspace, 256); a.ws_m = a.ws_acc + slots * D; a.ws_l = a.ws_m + slots;
    a.max_len = L->max_seq_len;
    hipStream_t st = as_stream(stream);
    e = L->dtype == RK_F32 ? (q8 ? launch_rows_q8_f32(a, p.per, st) : launch_rows_f32(a, p.per, st))
                           : (q8 ? launch_rows_q8_bf16(a, p.per, st) : launch_rows_bf16(a, p.per, st));
    if (e != hipSuccess) return hip_fail(ctx, e, "attention launch");
    if (p.Sv + p.Sr > 1) {
        e = launch_rows_merge(L->dtype, a, st);
        if (e != hipSuccess) return hip_fail(ctx, e, "attention merge launch");
    }
    return RK_OK;
}

rk_status rk_decode_attn_quant(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_q8, const void* v_q8,
                            const float* R_r, const float* delta_mu, const rk_text* text, float scale, void* out,
                            void* workspace, size_t workspace_bytes, void* stream)
{
    return rows_common(ctx, L, q, k_q8, v_q8, R_r, delta_mu, text, nullptr, true, scale, out, workspace, workspace_bytes, stream);
}

static rk_status tree_common(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_cache, const void* v_cache,
                             const float* R_r, const float* delta_mu, const rk_text* text, const rk_drafts* drafts, bool q8,
                             float scale, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    const rk_status s = check_drafts(ctx, drafts);
    return s != RK_OK ? s : rows_common(ctx, L, q, k_cache, v_cache, R_r, delta_mu, text, drafts, q8, scale, out, workspace,
                                        workspace_bytes, stream);
}

rk_status rk_decode_attn_tree(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_packed, const void* v_cache,
                              const float* R_r, const float* delta_mu, const rk_text* text, const rk_drafts* drafts,
                              float scale, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    return tree_common(ctx, L, q, k_packed, v_cache, R_r, delta_mu, text, drafts, false, scale, out, workspace, workspace_bytes, stream);
}

rk_status rk_decode_attn_tree_quant(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_q8, const void* v_q8,
                                 const float* R_r, const float* delta_mu, const rk_text* text, const rk_drafts* drafts,
                                 float scale, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    return tree_common(ctx, L, q, k_q8, v_q8, R_r, delta_mu, text, drafts, true, scale, out, workspace, workspace_bytes, stream);
}

rk_status rk_append_text_path(rk_ctx* ctx, const rk_layout* L, const rk_text* text, const rk_drafts* drafts,
                              const int32_t* path, int32_t path_len, const int32_t* n_path, int32_t* len_out, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK) return s;
    if (!text) return fail(ctx, RK_ERR_INVALID_ARG, "append_text_path: text is NULL");
    if ((s = check_text(ctx, text, true)) != RK_OK || (s = check_drafts(ctx, drafts)) != RK_OK) return s;
    if (!path || !n_path || !len_out) return fail(ctx, RK_ERR_INVALID_ARG, "append_text_path: NULL pointer (path, n_path, len_out)");
    if (path_len < 1 || path_len > RK_MAX_DRAFTS)
        return fail(ctx, RK_ERR_INVALID_ARG, "append_text_path: path_len %d outside 1..%d", path_len, RK_MAX_DRAFTS);
    if (text->max_len > text->capacity - path_len)
        return fail(ctx, RK_ERR_CAPACITY, "append_text_path: %d + %d rows exceed capacity %d", text->max_len, path_len, text->capacity);
    // rows copied by one work-group may be read by another: the drafts' rows and the segment's lie apart
    const size_t es = elem_size(L->dtype);
    auto span = [&](int64_t sb, int64_t sh, int64_t st, int rows) {
        return (size_t)((L->batch - 1) * sb + (L->n_kv_heads - 1) * sh + (int64_t)(rows - 1) * st + D) * es;
    };
    const size_t tb = span(text->stride_b, text->stride_h, text->stride_t, text->capacity);
    const size_t db = span(drafts->stride_b, drafts->stride_h, drafts->stride_t, drafts->n_tokens);
    if (ranges_meet(text->k, tb, drafts->k, db) || ranges_meet(text->k, tb, drafts->v, db) || ranges_meet(text->v, tb, drafts->k, db) ||
        ranges_meet(text->v, tb, drafts->v, db))
        return fail(ctx, RK_ERR_INVALID_ARG, "append_text_path: text segment and drafts overlap in memory");
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    const PathArgs a{text->k, text->v, text->stride_b, text->stride_h, text->stride_t, text->len, text->capacity,
                     drafts->k, drafts->v, drafts->stride_b, drafts->stride_h, drafts->stride_t, drafts->n_tokens_dev,
                     path, n_path, len_out, L->batch, L->n_kv_heads, drafts->n_tokens, path_len};
    e = launch_append_path(L->dtype, a, ctx->tickets, as_stream(stream));
    return e == hipSuccess ? RK_OK : hip_fail(ctx, e, "append_text_path launch");
}

// q and q_out together, or neither
static rk_status check_turned(rk_ctx* ctx, const rk_heads* x, const rk_heads* out, const char* name, int B, int H, int n)
{
    if (!x && !out) return RK_OK;
    const rk_status s = check_heads(ctx, x, name);
    return s != RK_OK ? s : check_result(ctx, out, name, B, H, n);
}

rk_status rk_rope(rk_ctx* ctx, const rk_layout* L, const rk_rotary* rope, int32_t n_tokens, const int32_t* n_tokens_dev, const rk_heads* q,
                  const rk_heads* q_out, const rk_heads* k, const rk_heads* k_out, uint32_t flags, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK || (s = check_rope_tokens(ctx, L, n_tokens)) != RK_OK || (s = check_rotary(ctx, rope)) != RK_OK) return s;
    if (!q && !q_out && !k && !k_out) return fail(ctx, RK_ERR_INVALID_ARG, "rope: neither q nor k");
    if ((s = check_turned(ctx, q, q_out, "rope: q or q_out", L->batch, L->n_q_heads, n_tokens)) != RK_OK) return s;
    if ((s = check_turned(ctx, k, k_out, "rope: k or k_out", L->batch, L->n_kv_heads, n_tokens)) != RK_OK) return s;
    if (flags & ~RK_ROPE_INVERSE) return fail(ctx, RK_ERR_INVALID_ARG, "rope: unknown flags %x", flags);
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    if (n_tokens == 0) return RK_OK;
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    RopeArgs a = rope_args(L, rope, n_tokens, n_tokens_dev);
    a.inverse = flags & RK_ROPE_INVERSE;
    if (q) {
        a.q = q->data; a.q_sb = q->stride_b; a.q_sh = q->stride_h; a.q_st = q->stride_t;
        a.qo = q_out->data; a.qo_sb = q_out->stride_b; a.qo_sh = q_out->stride_h; a.qo_st = q_out->stride_t;
    }
    if (k) {
        a.k = k->data; a.k_sb = k->stride_b; a.k_sh = k->stride_h; a.k_st = k->stride_t;
        a.ko = k_out->data; a.ko_sb = k_out->stride_b; a.ko_sh = k_out->stride_h; a.ko_st = k_out->stride_t;
    }
    e = launch_rope(L->dtype, a, nullptr, ctx->n_cu, as_stream(stream));
    return e == hipSuccess ? RK_OK : hip_fail(ctx, e, "rope launch");
}

rk_status rk_rope_append_text(rk_ctx* ctx, const rk_layout* L, const rk_rotary* rope, int32_t n_tokens, const int32_t* n_tokens_dev,
                              const rk_heads* q, const rk_heads* q_out, const rk_heads* k, const rk_heads* v, const rk_text* text,
                              int32_t* len_out, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK || (s = check_rope_tokens(ctx, L, n_tokens)) != RK_OK || (s = check_rotary(ctx, rope)) != RK_OK) return s;
    if (!text) return fail(ctx, RK_ERR_INVALID_ARG, "rope_append_text: text is NULL");
    if ((s = check_text(ctx, text, true)) != RK_OK) return s;
    if ((s = check_turned(ctx, q, q_out, "rope_append_text: q or q_out", L->batch, L->n_q_heads, n_tokens)) != RK_OK) return s;
    if ((s = check_heads(ctx, k, "rope_append_text: k")) != RK_OK || (s = check_heads(ctx, v, "rope_append_text: v")) != RK_OK) return s;
    if (!len_out) return fail(ctx, RK_ERR_INVALID_ARG, "rope_append_text: len_out is NULL");
    // (written while other work-groups may still read it)
    if (len_out == n_tokens_dev) return fail(ctx, RK_ERR_INVALID_ARG, "rope_append_text: len_out is n_tokens_dev");
    if (n_tokens < 1) return fail(ctx, RK_ERR_INVALID_ARG, "rope_append_text: n_tokens %d", n_tokens);
    if (text->max_len > text->capacity - n_tokens)
        return fail(ctx, RK_ERR_CAPACITY, "rope_append_text: %d + %d rows exceed capacity %d", text->max_len, n_tokens, text->capacity);
    // each row is written by a work-group of its own
    const rk_heads rows{text->k, text->stride_b, text->stride_h, text->stride_t};
    if (!rows_apart(&rows, L->batch, L->n_kv_heads, text->max_len + n_tokens))
        return fail(ctx, RK_ERR_INVALID_ARG, "rope_append_text: rows of the text segment share elements");
    // rows written by one work-group may be read by another: the segment's rows and the sources lie apart
    const size_t es = elem_size(L->dtype);
    const size_t tb = heads_bytes(text->stride_b, text->stride_h, text->stride_t, L->batch, L->n_kv_heads, text->capacity, es);
    for (const rk_heads* x : {k, v}) {
        const size_t xb = heads_bytes(x->stride_b, x->stride_h, x->stride_t, L->batch, L->n_kv_heads, n_tokens, es);
        if (ranges_meet(text->k, tb, x->data, xb) || ranges_meet(text->v, tb, x->data, xb))
            return fail(ctx, RK_ERR_INVALID_ARG, "rope_append_text: text segment and new rows overlap in memory");
    }
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    RopeArgs a = rope_args(L, rope, n_tokens, n_tokens_dev);
    if (q) {
        a.q = q->data; a.q_sb = q->stride_b; a.q_sh = q->stride_h; a.q_st = q->stride_t;
        a.qo = q_out->data; a.qo_sb = q_out->stride_b; a.qo_sh = q_out->stride_h; a.qo_st = q_out->stride_t;
    }
    a.k = k->data; a.k_sb = k->stride_b; a.k_sh = k->stride_h; a.k_st = k->stride_t;
    a.v = v->data; a.v_sb = v->stride_b; a.v_sh = v->stride_h; a.v_st = v->stride_t;
    a.ko = text->k; a.vo = text->v; a.ko_sb = text->stride_b; a.ko_sh = text->stride_h; a.ko_st = text->stride_t;
    a.len = text->len; a.cap = text->capacity; a.len_out = len_out;
    e = launch_rope(L->dtype, a, ctx->tickets, ctx->n_cu, as_stream(stream));
    return e == hipSuccess ? RK_OK : hip_fail(ctx, e, "rope_append_text launch");
}

size_t rk_window_workspace_size(const rk_ctx* ctx, const rk_layout* L, int32_t n_tokens)
{
    if (check_layout(nullptr, L) != RK_OK || n_tokens < 1 || n_tokens > RK_MAX_TOKENS) return 0;
    const size_t one = rows_ws(ctx, L, 1), many = prefill_ws(ctx, L, n_tokens);
    return one > many ? one : many;
}

rk_status rk_prefill_plan(const rk_ctx* ctx, const rk_layout* L, int32_t n_tokens, int32_t max_len, int32_t window, int32_t sinks,
                          int32_t* rows_per_work_group, int32_t* n_splits)
{
    rk_status s = check_layout(nullptr, L);
    if (s != RK_OK || (s = check_tokens(nullptr, L, n_tokens)) != RK_OK || (s = check_window(nullptr, window, sinks)) != RK_OK) return s;
    if (n_tokens < 1 || max_len < 0 || max_len > RK_MAX_TOKENS || !rows_per_work_group || !n_splits) return RK_ERR_INVALID_ARG;
    const PrefillPlan p = prefill_plan(ctx, L, n_tokens, max_len, window, sinks);
    if ((s = check_prefill_groups(nullptr, L, p)) != RK_OK) return s;
    *rows_per_work_group = p.rows;
    *n_splits = p.S;
    return RK_OK;
}

rk_status rk_prefill_attn_window(rk_ctx* ctx, const rk_layout* L, const rk_heads* q, int32_t n_tokens, const int32_t* n_tokens_dev,
                                 const rk_text* text, int32_t window, int32_t sinks, float scale, const rk_heads* out, void* workspace,
                                 size_t workspace_bytes, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK || (s = check_tokens(ctx, L, n_tokens)) != RK_OK || (s = check_window(ctx, window, sinks)) != RK_OK) return s;
    if (n_tokens < 1) return fail(ctx, RK_ERR_INVALID_ARG, "prefill_attn_window: n_tokens %d", n_tokens);
    if ((s = check_heads(ctx, q, "prefill_attn_window: q")) != RK_OK) return s;
    if ((s = check_result(ctx, out, "prefill_attn_window: out", L->batch, L->n_q_heads, n_tokens)) != RK_OK) return s;
    if (!text) return fail(ctx, RK_ERR_INVALID_ARG, "prefill_attn_window: text is NULL");
    if ((s = check_text(ctx, text, false)) != RK_OK) return s;
    if (text->max_len > RK_MAX_TOKENS) return fail(ctx, RK_ERR_INVALID_ARG, "prefill_attn_window: max_len exceeds %d", RK_MAX_TOKENS);
    const size_t need = prefill_ws(ctx, L, n_tokens);
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))
        return fail(ctx, RK_ERR_WORKSPACE, "prefill_attn_window workspace: need %zu bytes, 16-byte aligned", need);
    const PrefillPlan p = prefill_plan(ctx, L, n_tokens, text->max_len, window, sinks, text->stride_t);
    if ((s = check_prefill_groups(ctx, L, p)) != RK_OK) return s;
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    PrefillArgs a{};
    a.q = q->data; a.q_sb = q->stride_b; a.q_sh = q->stride_h; a.q_st = q->stride_t;
    a.out = out->data; a.o_sb = out->stride_b; a.o_sh = out->stride_h; a.o_st = out->stride_t;
    a.k = text->k; a.v = text->v; a.sb = text->stride_b; a.sh = text->stride_h; a.st = text->stride_t;
    a.len = text->len; a.max_len = text->max_len; a.n_dev = n_tokens_dev; a.n = n_tokens;
    a.B = L->batch; a.Hq = L->n_q_heads; a.Hkv = L->n_kv_heads; a.G = a.Hq / a.Hkv;
    a.window = window; a.sinks = sinks;
    a.rows = p.rows; a.blocks = p.blocks; a.S = p.S;
    for (int i = 0; i < PREFILL_CUTS; ++i) a.cut[i] = i + 1 >= p.S ? p.blocks : p.tokens ? prefill_cut(p.rows, a.G, n_tokens, text->max_len, (int64_t)(i + 1) * p.tokens) : 0;
    const float sc = scale > 0.f ? scale : 1.0f / sqrtf((float)L->head_dim);
    a.scale_log2 = sc * 1.44269504088896340736f;
    const size_t slots = (size_t)a.B * a.Hq * n_tokens * a.S;
    a.ws_acc = (float*)align_up((uintptr_t)workspace, 256); a.ws_m = a.ws_acc + slots * D; a.ws_l = a.ws_m + slots;
    e = launch_prefill(L->dtype, a, as_stream(stream));
    return e == hipSuccess ? RK_OK : hip_fail(ctx, e, "prefill_attn_window launch");
}

static rk_status window_common(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_cache, const void* v_cache, const float* R_r,
                               const float* delta_mu, const rk_text* text, int32_t window, int32_t sinks, bool q8, float scale, void* out,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    if (!ctx) return RK_ERR_INVALID_ARG;
    rk_status s = check_layout(ctx, L);
    if (s != RK_OK || (s = check_window(ctx, window, sinks)) != RK_OK) return s;
    const bool cache = k_cache || v_cache;
    if (!q || !out || (cache && (!k_cache || !v_cache || !R_r || !L->seq_len)))
        return fail(ctx, RK_ERR_INVALID_ARG, "attention: NULL pointer (q, out; one of the caches, R_r, seq_len)");
    if (((uintptr_t)k_cache & 15) || ((uintptr_t)v_cache & 15) || ((uintptr_t)q & 15))
        return fail(ctx, RK_ERR_INVALID_ARG, "attention: q and the caches must be 16-byte aligned");
    if (cache && L->max_seq_len > L->capacity)
        return fail(ctx, RK_ERR_CAPACITY, "attention: max_seq_len %d exceeds capacity %d", L->max_seq_len, L->capacity);
    if (!text) return fail(ctx, RK_ERR_INVALID_ARG, "decode_attn_window: text is NULL");
    if ((s = check_text(ctx, text, false)) != RK_OK) return s;
    if (text->max_len > RK_MAX_TOKENS) return fail(ctx, RK_ERR_INVALID_ARG, "decode_attn_window: max_len exceeds %d", RK_MAX_TOKENS);
    if ((int64_t)L->batch * L->n_q_heads > INT32_MAX) return fail(ctx, RK_ERR_UNSUPPORTED, "attention: more than %d query rows", INT32_MAX);
    const size_t need = rows_ws(ctx, L, 1);
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15))
        return fail(ctx, RK_ERR_WORKSPACE, "attention workspace: need %zu bytes, 16-byte aligned", need);
    const RowsPlan p = window_plan(ctx, L, cache, window_rows(text->max_len, window, sinks), q8);
    if ((s = check_rows_groups(ctx, L, p)) != RK_OK) return s;
    if (ctx->device == RK_DEVICE_NONE) return fail(ctx, RK_ERR_NO_DEVICE, "valid arguments, but the context has no device");
    DeviceGuard dev(ctx->device);
    hipError_t e = dev.status;
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    WindowRowsArgs a{};
    a.q = q; a.Kc = k_cache; a.Vc = v_cache; a.Rr = R_r; a.dmu = delta_mu; a.seq_len = L->seq_len; a.out = out;
    a.B = L->batch; a.T = 1; a.Hq = L->n_q_heads; a.Hkv = L->n_kv_heads; a.G = a.Hq / a.Hkv;
    a.cap = L->capacity; a.r = L->keep; a.rp = keep_padded(L->keep);
    a.Sv = p.Sv; a.Sr = p.Sr; a.nrb = p.nrb;
    const float sc = scale > 0.f ? scale : 1.0f / sqrtf((float)L->head_dim);
    a.scale_log2 = sc * 1.44269504088896340736f;
    a.text_k = text->k; a.text_v = text->v; a.text_len = text->len; a.text_max = text->max_len;
    a.text_sb = text->stride_b; a.text_sh = text->stride_h; a.text_st = text->stride_t;
    const size_t slots = (size_t)a.B * a.Hq * (p.Sv + p.Sr);
    a.ws_acc = (float*)align_up((uintptr_t)workspace, 256); a.ws_m = a.ws_acc + slots * D; a.ws_l = a.ws_m + slots;
    a.max_len = L->max_seq_len;
    a.window = window; a.sinks = sinks;
    hipStream_t st = as_stream(stream);
    e = L->dtype == RK_F32 ? (q8 ? launch_window_rows_q8_f32(a, st) : launch_window_rows_f32(a, st))
                           : (q8 ? launch_window_rows_q8_bf16(a, st) : launch_window_rows_bf16(a, st));
    if (e != hipSuccess) return hip_fail(ctx, e, "attention launch");
    if (p.Sv + p.Sr > 1) {
        e = launch_rows_merge(L->dtype, a, st);
        if (e != hipSuccess) return hip_fail(ctx, e, "attention merge launch");
    }
    return RK_OK;
}

rk_status rk_decode_attn_window(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_packed, const void* v_cache, const float* R_r,
                                const float* delta_mu, const rk_text* text, int32_t window, int32_t sinks, float scale, void* out,
                                void* workspace, size_t workspace_bytes, void* stream)
{
    return window_common(ctx, L, q, k_packed, v_cache, R_r, delta_mu, text, window, sinks, false, scale, out, workspace, workspace_bytes, stream);
}

rk_status rk_decode_attn_window_quant(rk_ctx* ctx, const rk_layout* L, const void* q, const void* k_q8, const void* v_q8, const float* R_r,
                                      const float* delta_mu, const rk_text* text, int32_t window, int32_t sinks, float scale, void* out,
                                      void* workspace, size_t workspace_bytes, void* stream)
{
    return window_common(ctx, L, q, k_q8, v_q8, R_r, delta_mu, text, window, sinks, true, scale, out, workspace, workspace_bytes, stream);
}

}  // extern "C"
