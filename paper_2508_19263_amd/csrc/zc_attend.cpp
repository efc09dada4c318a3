// Host side of the operators over K/V pages: argument checks, the choice of kernels and splits, and the C entry points
// zc_attend, zc_attend_shared, zc_attend_workspace_bytes, zc_kv_write, zc_kv_read and zc_evict.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>

#include "zc_attend.h"
#include "zc_host.h"

namespace zc {

namespace {

constexpr uint32_t kMaxTokens = 1u << 30;      // positions are signed 32-bit numbers in the kernels, sums of two included
constexpr uint64_t kMaxBlocks = (1u << 24) - 1;   // of 256 threads: HIP launches fewer than 2^32
constexpr uint32_t kMaxSlots = 64;             // parts of one row: k_attend_join holds one per lane
constexpr uint64_t kMostLogits = 1u << 30;     // bytes of scratch

bool aligned4(const void *p) { return ((uintptr_t)p & 3) == 0; }

bool fp4(uint32_t format) { return format == ZC_FMT_FP4_E2M1_MX || format == ZC_FMT_FP4_E2M1_NV; }
uint32_t row_bytes(const zc_kv_cache &c) { return c.format == ZC_FMT_BF16 ? c.head_dim * 2 : fp4(c.format) ? c.head_dim / 2 : c.head_dim; }
uint32_t row_scales(const zc_kv_cache &c) { return !fp4(c.format) ? 0 : c.head_dim / (c.format == ZC_FMT_FP4_E2M1_MX ? 32 : 16); }

zc_status check_cache(const zc_kv_cache *c, PagesDev *out)
{
    if (!c) return ZC_ERR_INVALID_ARG;
    constexpr uint32_t kFirstLayout = offsetof(zc_kv_cache, d_k_block_scales);
    if (c->struct_size != sizeof(zc_kv_cache) && c->struct_size != kFirstLayout) return ZC_ERR_UNSUPPORTED;
    if (c->format != ZC_FMT_BF16 && c->format != ZC_FMT_FP8_E4M3 && c->format != ZC_FMT_FP8_E5M2 && !fp4(c->format)) return ZC_ERR_UNSUPPORTED;
    void *const k_blocks = c->struct_size == kFirstLayout ? nullptr : c->d_k_block_scales, *const v_blocks = c->struct_size == kFirstLayout ? nullptr : c->d_v_block_scales;
    if (fp4(c->format) ? !k_blocks || !v_blocks : k_blocks || v_blocks) return ZC_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return ZC_ERR_UNSUPPORTED;
    if (c->page_tokens < 16 || c->page_tokens > 65536 || (c->page_tokens & (c->page_tokens - 1))) return ZC_ERR_INVALID_ARG;
    if (!c->n_seqs || !c->n_heads || !c->table_pages || !c->n_pages || c->n_pages > 0x7FFFFFFFu) return ZC_ERR_INVALID_ARG;
    const uint64_t capacity = (uint64_t)c->table_pages * c->page_tokens;
    if (capacity >= kMaxTokens || (uint64_t)c->n_seqs * c->n_heads > (kMaxBlocks >> 2)) return ZC_ERR_INVALID_ARG;     // (k_evict_select has 1,024 threads for each)
    if (!c->d_k_pages || !c->d_v_pages || !c->d_table || !c->d_lengths) return ZC_ERR_INVALID_ARG;
    if (!aligned16(c->d_k_pages) || !aligned16(c->d_v_pages) || !aligned16(k_blocks) || !aligned16(v_blocks) || !aligned4(c->d_table) || !aligned4(c->d_lengths) ||
        !aligned4(c->d_k_scales) || !aligned4(c->d_v_scales)) return ZC_ERR_INVALID_ARG;
    PagesDev d = {};
    d.k = (const uint8_t *)c->d_k_pages;
    d.v = (const uint8_t *)c->d_v_pages;
    d.k_blocks = (const uint8_t *)k_blocks;
    d.v_blocks = (const uint8_t *)v_blocks;
    d.table = c->d_table;
    d.lengths = c->d_lengths;
    d.k_scales = c->d_k_scales;
    d.v_scales = c->d_v_scales;
    d.heads = c->n_heads;
    d.table_pages = c->table_pages;
    d.n_pages = c->n_pages;
    while ((1u << d.page_shift) < c->page_tokens) d.page_shift++;
    d.capacity = d.limit = (int32_t)capacity;
    *out = d;
    return ZC_OK;
}

bool same_shape(const zc_kv_cache &a, const zc_kv_cache &b) { return a.format == b.format && a.n_heads == b.n_heads && a.head_dim == b.head_dim; }

// one pass over a cache: k_attend_many with tiles x 128 rows to a workgroup, or k_attend_few with tiles x 16
struct Pass {
    bool many;
    uint32_t tiles, row_blocks, even, splits, long_part;
    bool eight;                                // k_attend_short
    uint64_t blocks;
};

// rows: of one (sequence, head), or of one head of the prefix; units: how many of those; longest: tokens that a row block may have to read;
// only: the call has no other pass
Pass plan_pass(uint64_t rows, uint64_t units, uint64_t longest, uint32_t most_splits, bool only, bool fp4, bool weights)
{
    Pass p;
    // k_attend_few goes over a cache once for every 32 rows, k_attend_many once for 128.  Microseconds of the former against the latter, rows to a
    // K/V head in front, one query head each, 8 K/V heads: 64: 4 FP8 caches of 8,192 tokens 25.7 against 30.4, one 15.7 against 19.6, 4 BF16 ones
    // of 4,000 21.3 against 27.0, six E5M2 ones with heads of 64 and a window of 2,048 15.8 against 19.8, 16 BF16 ones of 1,000 with heads of 64
    // 13.6 against 18.2; 65 (a third row block): 39.1 against 31.7, 18.3 against 19.8, 34.6 against 28.0, 17.6 against 20.3, 18.2 against 18.6.
    // Where caches alone fill the GPU the boundary lies lower, for BF16 below 33: 32 BF16 ones of 4,000 147 against 106 (33 rows) and 151 against 111
    // (64), 32 FP8 ones of 8,192 141 against 136 (35) and 145 against 140 (64).
    p.many = rows > 64;
    p.tiles = p.many || rows <= 16 ? 1 : 2;
    const uint64_t per_block = p.tiles * (p.many ? 128 : 16);
    p.row_blocks = (uint32_t)((rows + per_block - 1) / per_block);
    // A cache is split where there are fewer workgroups than compute units (k_attend_many: two of whose workgroups share one), but
    // into parts of no less than two steps of 128 tokens (four of 64).  Measured with one workgroup per compute unit against two in
    // k_attend_few: 4 FP8 caches of 8,192 tokens 17.6 against 18.3 us, 32 BF16 ones with a window of 4,096 94 against 100 us; with
    // parts of two steps against four: one cache with a window of 512 9.0 against 9.6 us, 1,531 shared tokens 19.1 against 21.4 us.
    // A call's only pass is left in one part up to 640 tokens: a second launch costs what its part of the work takes.
    const uint64_t groups = units * p.row_blocks, part = 256;
    // FP4, up to a workgroup for each compute unit: k_attend_short, whose eight wavefronts take what four of k_attend_few and a join take longer for.
    // Microseconds of calls one after the other, those against it, 8 K/V heads of 128, 4 query heads to each: one MXFP4 cache of 260 tokens 6.4 and 6.1, 640
    // 7.5 and 7.0, 700 8.6 and 7.9, 1,000 9.0 and 8.8, 1,280 8.7 and 9.5; NVFP4 640 8.6 and 7.7, 1,000 9.1 and 10.3 (from Python, which takes longer for two
    // launches and scratch than the GPU does, 15 and 11); 32 MXFP4 ones of 1,000 12.7 and 9.7, 2,048 18.1 and 15.6, NVFP4 19.2 and 17.0.  (128 tokens 5.2 and 5.5.)
    const bool may_be_eight = fp4 && only && !weights && rows <= 16 && groups <= 256;
    const uint64_t one_part = !may_be_eight ? 640 : groups <= 128 ? 1024 : 2048, possible = only && longest <= one_part ? 1 : (longest + part - 1) / part;
    // Lengths are not known here, only the longest.  So that one long cache among short ones does not keep everyone waiting, parts are at
    // most kLongPart tokens, and what is left over of a shorter cache's parts ends at once: 31 FP8 caches of 1,000 tokens and one of 131,072
    // 1,077 -> 128 us, 64 of 0 to 32,768 444 -> 408 us; 64 of 8,192 188 us as before, 16 of 32,768 190 -> 198 us.  (At most 4,096: 109, 391,
    // 202 and 209 us.)  k_attend_many has row blocks enough where rows are many, and its parts would take their number times as much room.
    // A part of an FP4 cache is half the bytes and nearly as much work, and a compute unit takes up to four of its workgroups: parts of at most 4,096
    // tokens, and two for each compute unit where rows fill one tile.  Microseconds of one workgroup and 8,192 tokens, against 512 and 4,096 (MX, 8
    // K/V heads of 128, 4 query heads to each): one cache of 131,072 tokens 48.0 and 38.7, 8 of 8,192 23.9 and 20.6, 24 of 15,005 98 and 86, 24 of 0 to
    // 30,011 114 and 97, 64 of 0 to 32,768 264 and 238; 32 of 16,384 113.9 and 114.6; of 32 rows each, 4 of 8,192 21.8 and 23.1.
    // Where rows fill one tile and there are fewer than two (sequence, head)s for each compute unit, whose parts end at very different times, parts are of at
    // most 2,560 tokens.  Microseconds of 4,096 against 2,560: 24 NVFP4 caches of 0 to 30,011 94.4 and 91.1, with weights 130 and 127, 17 of 0 to 23,302
    // 75.5 and 56.1, 16 of 16,384 62.0 and 58.9; 17 MXFP4 ones of 0 to 29,067 84.9 and 62.9, of 17,109 72.5 and 64.8, 40 of 8,348 74.5 and 66.8, but 32 of 16,384 99.1 and 102.9, 40 of 3,000 to 20,000 100 and
    // 107; where there are more: 64 NVFP4 ones of 0 to 5,606 52.2 and 54.7, MXFP4 of 8,192 99.4 and 103.3, of 0 to 6,576 56.5 and 54.9;
    // seven NVFP4 ones of 3,000 to 20,000, 64 rows, 69 and 77.  (2,048: those of 16,384 105 and, NV, 63.)
    p.long_part = !fp4 ? kLongPart : p.tiles == 1 && groups < 512 ? kShortPart : kLongPart / 2;
    const uint64_t enough = p.many || (fp4 && p.tiles == 1) ? 512 : 256;
    uint64_t even = groups ? (enough + groups - 1) / groups : 1;
    if (even > possible) even = possible;
    if (even > most_splits) even = most_splits;
    if (!even) even = 1;
    const uint64_t least = p.many ? 1 : (longest + p.long_part - 1) / p.long_part, s = even > least ? even : least;
    p.even = (uint32_t)even;
    p.splits = (uint32_t)(s < most_splits ? s : most_splits);
    p.eight = may_be_eight && p.splits == 1 && longest > 256;
    p.blocks = groups * p.splits;
    return p;
}

int launch_pass(const AttendDev &a, const Pass &p, const zc_kv_cache &c, void *stream)
{
    return p.many ? launch_attend_many(a, c.format, c.head_dim, stream) : launch_attend_few(a, c.format, c.head_dim, p.tiles, stream);
}

// a call's passes and workspace, from its arguments
struct AttendPlan {
    AttendDev own;
    AttendDev pre;
    Pass own_pass, pre_pass;
    uint32_t slots;                            // 1: the only pass writes the result itself
    uint64_t part_o_bytes, logits_at, weights_at, ws_bytes;
    uint32_t weight_parts;
    bool logits;                               // weights come from the logits that the pass leaves, else from the keys again
};

zc_status plan_attend(const zc_attend_args *x, const zc_kv_cache *prefix, const zc_kv_cache *cache, bool shared, AttendPlan *out)
{
    if (!x || !cache || (shared && !prefix)) return ZC_ERR_INVALID_ARG;
    if (x->struct_size != sizeof(zc_attend_args)) return ZC_ERR_UNSUPPORTED;
    AttendPlan p = {};
    AttendDev &a = p.own;
    zc_status st = check_cache(cache, &a.c);
    if (st) return st;
    if (!x->n_q_heads || x->n_q_heads % cache->n_heads || !x->max_q_len) return ZC_ERR_INVALID_ARG;
    if (!x->d_q_start && (x->n_tokens != cache->n_seqs)) return ZC_ERR_INVALID_ARG;
    if ((uint64_t)x->n_tokens * x->n_q_heads > 0x3FFFFFFFu || x->max_q_len >= kMaxTokens) return ZC_ERR_INVALID_ARG;
    if (x->n_tokens && (!x->d_q || !x->d_out)) return ZC_ERR_INVALID_ARG;
    if (!aligned16(x->d_q) || !aligned16(x->d_out) || !aligned4(x->d_q_start) || !aligned4(x->d_lse) || !aligned4(x->d_weights_in) ||
        !aligned4(x->d_weights_out)) return ZC_ERR_INVALID_ARG;
    if ((x->q_token_stride | x->q_head_stride | x->out_token_stride | x->out_head_stride) & 7) return ZC_ERR_INVALID_ARG;
    if (!std::isfinite(x->scale) || x->reserved) return ZC_ERR_INVALID_ARG;
    if (x->d_weights_out && (shared || (x->n_tokens && !x->d_lse))) return ZC_ERR_INVALID_ARG;
    if (x->d_weights_in && !x->d_weights_out) return ZC_ERR_INVALID_ARG;
    if (x->d_weights_out && x->n_tokens && x->d_out == x->d_q) return ZC_ERR_INVALID_ARG;       // (k_attend_weights reads the queries when the results are there)
    if (x->max_kv_len && x->max_kv_len < (uint32_t)a.c.limit) a.c.limit = (int32_t)x->max_kv_len;

    a.q = (const uint16_t *)x->d_q;
    a.out = (uint16_t *)x->d_out;
    a.lse = x->d_lse;
    a.q_start = x->d_q_start;
    a.own_lengths = cache->d_lengths;
    a.q_token_stride = x->q_token_stride;
    a.q_head_stride = x->q_head_stride;
    a.out_token_stride = x->out_token_stride;
    a.out_head_stride = x->out_head_stride;
    a.scale = x->scale;
    a.own_limit = a.c.limit;
    a.n_seqs = cache->n_seqs;
    a.n_tokens = x->n_tokens;
    a.q_heads = x->n_q_heads;
    a.group = x->n_q_heads / cache->n_heads;
    a.max_q_len = x->d_q_start ? (x->max_q_len < x->n_tokens ? x->max_q_len : x->n_tokens) : 1;
    a.window = x->window < kMaxTokens ? x->window : 0;
    a.sinks = x->sinks < kMaxTokens ? x->sinks : kMaxTokens;

    auto reach = [&](int32_t limit) {          // tokens of a cache that the rows of one sequence may see
        const uint64_t w = a.window ? (uint64_t)a.window + a.max_q_len + a.sinks + 64 : (uint64_t)limit;
        return w < (uint64_t)limit ? w : (uint64_t)limit;
    };
    p.own_pass = plan_pass((uint64_t)a.max_q_len * a.group, (uint64_t)a.n_seqs * a.c.heads, reach(a.c.limit), shared ? 16 : kMaxSlots, !shared, fp4(cache->format), x->d_weights_out);
    p.slots = p.own_pass.splits;
    if (shared) {
        AttendDev &b = p.pre;
        PagesDev pc;
        st = check_cache(prefix, &pc);
        if (st) return st;
        if (prefix->n_seqs != 1 || !same_shape(*prefix, *cache)) return ZC_ERR_INVALID_ARG;
        if (x->max_prefix_len && x->max_prefix_len < (uint32_t)pc.limit) pc.limit = (int32_t)x->max_prefix_len;
        if ((uint64_t)pc.limit + (uint64_t)a.c.limit >= kMaxTokens) return ZC_ERR_INVALID_ARG;
        a.prefix_length = prefix->d_lengths;
        a.prefix_limit = pc.limit;
        b = a;
        b.c = pc;
        b.shared = 1;
        p.pre_pass = plan_pass((uint64_t)a.n_tokens * a.group, a.c.heads, (uint64_t)pc.limit, 48, false, fp4(cache->format), false);
        b.splits = p.pre_pass.splits;
        b.even = p.pre_pass.even;
        b.long_part = p.pre_pass.long_part;
        b.row_blocks = p.pre_pass.row_blocks;
        b.first_slot = 0;
        a.first_slot = b.splits;
        p.slots += b.splits;
    } else if (x->max_prefix_len) return ZC_ERR_INVALID_ARG;
    a.splits = p.own_pass.splits;
    a.even = p.own_pass.even;
    a.long_part = p.own_pass.long_part;
    a.row_blocks = p.own_pass.row_blocks;
    a.direct = p.slots == 1;
    a.eight = p.own_pass.eight;
    // Pages that are read once and are more than the memory-side cache holds go past the caches.  Microseconds of a decoding step through them against
    // past them (8 K/V heads of 128): 64 caches of 8,192 tokens BF16 361 and 320, FP8 186 and 167, MXFP4 113 and 103, NVFP4 124 and 113; 200 FP8 ones of 2,000
    // 151 and 138, 24 of 0 to 30,011 160 and 167; 32 MXFP4 ones (285 MB) 60 and 57; 16 (142 MB) 33 and 32, 8 of MXFP4 20 and 21.5, 4 FP8 ones 16.6 and 18.6,
    // which find them there again.  Rows of less than 64 bytes lie four to a line that several loads take parts of: 64 MXFP4 caches of 16,384 tokens, 64
    // dimensions, 134 and 140.
    // The host knows the room and the pools, and a pool that the caches hold is never read past them.  BF16 and FP8 go on by the lengths and the table, on the
    // device (past_caches): 4 caches of 8,192 tokens in tables for 131,072, BF16 25.7 us through the caches and 27.0 past them, FP8 16.6 and 17.5; 64 of 8,192
    // that have their first 8,000 in the same pages BF16 145 and 188, FP8 89 and 95, the first 6,144 BF16 189 and 213, FP8 104 and 113, the first 4,096 BF16 243
    // and 241, FP8 139 and 131.  The choice takes two loads one after the other, which parts of less than kLeastChoice tokens do without: 4,000 BF16 caches
    // of 250 tokens 743 us through the caches, 779 past them, 877 with a choice for each, 2,000 of 500 716, 665 and 707, 1,200 of 800 670, 611 and 620, 1,000 of
    // 1,000 696, 633 and 636; FP8 405, 418 and 503; 375, 373 and 403; 349, 328 and 338; 359, 338 and 345.  FP4 goes by the room: its parts end sooner (with a choice 200
    // caches of 2,000 MXFP4 81.5 -> 84.4 us, NVFP4 88.8 -> 92.7, 24 of 0 to 30,011 88.9 -> 92.3 and 92.8 -> 96.5), and 4 of 8,192 in too much room lose no more
    // (MXFP4 13.2 and 13.8, NVFP4 14.6 and 15.0), 64 of 8,192 that share 6,144 a tenth (68 and 75, 91 and 98).
    const uint64_t held = kMemorySideCache / ((uint64_t)a.c.heads * 2 * (row_bytes(*cache) + row_scales(*cache)));       // tokens
    a.reach = (int32_t)reach(a.c.limit);
    if (!p.own_pass.many && p.own_pass.row_blocks == 1 && row_bytes(*cache) >= kLeastPast && (uint64_t)a.n_seqs * (uint64_t)a.reach > held &&
        (fp4(cache->format) || a.reach >= kLeastChoice) &&
        ((uint64_t)a.c.n_pages << a.c.page_shift) > held * a.c.heads) a.past_caches = held ? (uint32_t)held : 1;
    if (p.own_pass.blocks + p.pre_pass.blocks > kMaxBlocks) return ZC_ERR_INVALID_ARG;
    if (p.slots > 1) {
        const uint64_t rows = (uint64_t)a.n_tokens * a.q_heads * p.slots;
        p.part_o_bytes = rows * cache->head_dim * 4;
        p.ws_bytes = p.part_o_bytes + align256(rows * 8);
    }
    // Weights of few rows come from logits that the pass leaves (written and read again, 8 bytes per row and token), of more from
    // the keys again.  Microseconds from logits against keys, 32 caches of 8,000 tokens, 8 heads: 4 rows, FP8, 128 dimensions 134
    // against 233, 64 dimensions 79 against 153; 24 rows 190 against 235 and 145 against 164; 32 rows 216 against 229 and 176 against 161.
    // One cache of 4,000: 4 rows 11.8 against 17.6, 24 rows 20.1 against 20.8, 32 rows 22.5 against 20.8.
    // Logits have room for the longest length of every sequence, which large tables over few pages make much more than there are tokens, so
    // where they would take more than kMostLogits the keys are read again too (64 caches of 8,000 tokens, 4 rows, 128 dimensions, with room for
    // just 1 GiB of logits and for a step more: FP8 321 and 600 us, BF16 521 and 822; with max_kv_len = 8,000, 253 and 451).
    const uint64_t rows_per_head = (uint64_t)a.max_q_len * a.group, logit_stride = ((uint64_t)a.c.limit + 31) / 32 * 32;
    p.logits = x->d_weights_out && x->n_tokens && rows_per_head <= kLogitRows &&
               (uint64_t)a.n_seqs * a.c.heads * rows_per_head * logit_stride * 4 <= kMostLogits;
    if (p.logits) {
        a.logit_rows = (uint32_t)rows_per_head;
        a.logit_stride = (uint32_t)logit_stride;
        p.logits_at = p.ws_bytes = align256(p.ws_bytes);
        p.ws_bytes += (uint64_t)a.n_seqs * a.c.heads * a.logit_rows * a.logit_stride * 4;
    }
    const uint64_t join_blocks = (p.slots > 1 ? (uint64_t)a.n_tokens * a.q_heads : 0) + (p.logits ? (uint64_t)a.n_seqs * a.c.heads * (((uint64_t)a.c.limit + 1023) / 1024) : 0);
    if (join_blocks > kMaxBlocks) return ZC_ERR_INVALID_ARG;
    p.weight_parts = 1;
    if (x->d_weights_out && !p.logits) {
        // about 1,024 workgroups, of two that share a compute unit: a prompt's first tokens have the most rows, and the last ones fill up
        const uint64_t units = (uint64_t)a.n_seqs * a.c.heads, groups = units * ((uint64_t)(a.c.limit + 255) / 256);
        uint64_t parts = (1024 + groups - 1) / groups;
        if (parts > rows_per_head / 64) parts = rows_per_head / 64;
        if (parts > kMostParts) parts = kMostParts;
        p.weight_parts = parts ? (uint32_t)parts : 1;
        if (groups * p.weight_parts > kMaxBlocks) return ZC_ERR_INVALID_ARG;
        if (p.weight_parts > 1) {
            p.weights_at = align256(p.ws_bytes);
            p.ws_bytes = p.weights_at + units * p.weight_parts * (uint64_t)a.c.limit * 4;
        }
    }
    *out = p;
    return ZC_OK;
}

zc_status plan_rows(const zc_kv_rows *x, const zc_kv_cache *cache, RowsDev *out)
{
    if (!x || !cache) return ZC_ERR_INVALID_ARG;
    if (x->struct_size != sizeof(zc_kv_rows)) return ZC_ERR_UNSUPPORTED;
    RowsDev r = {};
    const zc_status st = check_cache(cache, &r.c);
    if (st) return st;
    if (!x->d_q_start && x->n_tokens != cache->n_seqs) return ZC_ERR_INVALID_ARG;
    // (at least 8,192 elements of a head to a workgroup where there are many)
    if ((uint64_t)x->n_tokens * cache->n_heads > 0x3FFFFFFFu || ((uint64_t)x->n_tokens * cache->head_dim + 8191) / 8192 * cache->n_heads > kMaxBlocks) return ZC_ERR_INVALID_ARG;
    if (x->n_tokens && (!x->d_k || !x->d_v)) return ZC_ERR_INVALID_ARG;
    if (!aligned16(x->d_k) || !aligned16(x->d_v) || !aligned4(x->d_q_start)) return ZC_ERR_INVALID_ARG;
    if ((x->k_token_stride | x->k_head_stride | x->v_token_stride | x->v_head_stride) & 7) return ZC_ERR_INVALID_ARG;
    r.k_pages = (uint8_t *)cache->d_k_pages;
    r.v_pages = (uint8_t *)cache->d_v_pages;
    r.k_scale_pages = const_cast<uint8_t *>(r.c.k_blocks);
    r.v_scale_pages = const_cast<uint8_t *>(r.c.v_blocks);
    r.k = (uint16_t *)x->d_k;
    r.v = (uint16_t *)x->d_v;
    r.k_token_stride = x->k_token_stride;
    r.k_head_stride = x->k_head_stride;
    r.v_token_stride = x->v_token_stride;
    r.v_head_stride = x->v_head_stride;
    r.q_start = x->d_q_start;
    r.n_seqs = cache->n_seqs;
    r.n_tokens = x->n_tokens;
    *out = r;
    return ZC_OK;
}

zc_status attend(const zc_attend_args *x, const zc_kv_cache *prefix, const zc_kv_cache *cache, bool shared, void *d_ws, uint64_t ws_bytes, void *stream)
{
    AttendPlan p;
    zc_status st = plan_attend(x, prefix, cache, shared, &p);
    if (st) return st;
    if (p.ws_bytes) {
        if (!d_ws || !aligned16(d_ws)) return ZC_ERR_INVALID_ARG;
        if (ws_bytes < p.ws_bytes) return ZC_ERR_BUFFER_TOO_SMALL;
        p.own.part_o = p.pre.part_o = (float *)d_ws;
        p.own.part_ml = p.pre.part_ml = (float *)((uint8_t *)d_ws + p.part_o_bytes);
        p.own.logits = p.logits ? (float *)((uint8_t *)d_ws + p.logits_at) : nullptr;
    }
    const WeightsDev w = {x->d_weights_in, x->d_weights_out, p.weight_parts > 1 ? (float *)((uint8_t *)d_ws + p.weights_at) : nullptr, p.weight_parts};
    if (x->n_tokens) {
        if (shared && !p.own_pass.many) {
            const uint32_t tiles = p.pre_pass.many || p.own_pass.tiles > p.pre_pass.tiles ? p.own_pass.tiles : p.pre_pass.tiles;
            LAUNCH_TRY(launch_attend_shared(p.pre, p.own, cache->format, cache->head_dim, p.pre_pass.many, tiles, stream));
        } else {
            if (shared) LAUNCH_TRY(launch_pass(p.pre, p.pre_pass, *cache, stream));
            LAUNCH_TRY(launch_pass(p.own, p.own_pass, *cache, stream));
        }
        if (p.slots > 1 || p.logits) LAUNCH_TRY(launch_attend_join(p.own, w, cache->head_dim, p.slots, stream));
    }
    if (x->d_weights_out && !p.logits) LAUNCH_TRY(launch_attend_weights(p.own, w, cache->format, cache->head_dim, stream));
    return ZC_OK;
}

}  // namespace

}  // namespace zc

extern "C" uint64_t zc_attend_workspace_bytes(const zc_attend_args *args, const zc_kv_cache *prefix, const zc_kv_cache *cache)
{
    zc::AttendPlan p;
    return zc::plan_attend(args, prefix, cache, prefix != nullptr, &p) ? 0 : p.ws_bytes;
}

extern "C" zc_status zc_attend(const zc_attend_args *args, const zc_kv_cache *cache, void *d_ws, uint64_t ws_bytes, void *stream)
{
    return zc::attend(args, nullptr, cache, false, d_ws, ws_bytes, stream);
}

extern "C" zc_status zc_attend_shared(const zc_attend_args *args, const zc_kv_cache *prefix, const zc_kv_cache *cache, void *d_ws, uint64_t ws_bytes, void *stream)
{
    return zc::attend(args, prefix, cache, true, d_ws, ws_bytes, stream);
}

extern "C" zc_status zc_kv_write(const zc_kv_rows *rows, const zc_kv_cache *cache, void *stream)
{
    zc::RowsDev r;
    const zc_status st = zc::plan_rows(rows, cache, &r);
    if (st) return st;
    // (K and V have the same page numbers: in one pool they would overwrite each other, unless they are the same bits)
    const bool tied = r.k == r.v && r.k_token_stride == r.v_token_stride && r.k_head_stride == r.v_head_stride && r.c.k_scales == r.c.v_scales;
    const bool one_pool = r.k_pages == r.v_pages, one_scale_pool = r.k_scale_pages && r.k_scale_pages == r.v_scale_pages;
    if (!tied && (one_pool || one_scale_pool)) return ZC_ERR_INVALID_ARG;
    if (r.n_tokens) LAUNCH_TRY(zc::launch_kv_write(r, cache->format, cache->head_dim, stream));
    return ZC_OK;
}

extern "C" zc_status zc_kv_read(const zc_kv_rows *rows, const zc_kv_cache *cache, void *stream)
{
    zc::RowsDev r;
    const zc_status st = zc::plan_rows(rows, cache, &r);
    if (st) return st;
    if (r.n_tokens && r.k == r.v) return ZC_ERR_INVALID_ARG;
    if (r.n_tokens) LAUNCH_TRY(zc::launch_kv_read(r, cache->format, cache->head_dim, stream));
    return ZC_OK;
}

extern "C" zc_status zc_evict(const zc_kv_cache *from, const float *d_weights, uint32_t keep, uint32_t sinks, uint32_t recent,
                              const zc_kv_cache *to, float *d_weights_to, int32_t *d_kept, void *stream)
{
    zc::EvictDev e = {};
    zc_status st = zc::check_cache(from, &e.from);
    if (!st) st = zc::check_cache(to, &e.to);
    if (st) return st;
    if (!zc::same_shape(*from, *to) || from->n_seqs != to->n_seqs || from->d_lengths == to->d_lengths) return ZC_ERR_INVALID_ARG;
    // (keys and values that lie apart would overwrite each other in one pool)
    if (to->d_k_pages == to->d_v_pages && from->d_k_pages != from->d_v_pages) return ZC_ERR_INVALID_ARG;
    if (e.to.k_blocks && e.to.k_blocks == e.to.v_blocks && e.from.k_blocks != e.from.v_blocks) return ZC_ERR_INVALID_ARG;
    if (!d_weights || (keep && !d_kept) || !zc::aligned4(d_weights) || !zc::aligned4(d_weights_to) || !zc::aligned4(d_kept)) return ZC_ERR_INVALID_ARG;
    if (d_weights_to == d_weights || (uint64_t)sinks + recent > keep || keep >= zc::kMaxTokens) return ZC_ERR_INVALID_ARG;
    const uint64_t most = keep < (uint32_t)e.from.capacity ? keep : (uint32_t)e.from.capacity;     // rows per sequence and head
    if (to->table_pages * (uint64_t)to->page_tokens < most) return ZC_ERR_BUFFER_TOO_SMALL;
    if ((uint64_t)from->n_seqs * from->n_heads * ((most + 63) / 64) > zc::kMaxBlocks) return ZC_ERR_INVALID_ARG;
    e.k_to = (uint8_t *)to->d_k_pages;
    e.v_to = (uint8_t *)to->d_v_pages;
    e.weights = d_weights;
    e.weights_to = d_weights_to;
    e.kept = d_kept;
    e.lengths_to = to->d_lengths;
    e.n_seqs = from->n_seqs;
    e.keep = keep;
    e.sinks = sinks;
    e.recent = recent;
    e.row_bytes = zc::row_bytes(*from);
    e.row_scales = zc::row_scales(*from);
    if (e.row_scales) {
        e.k_blocks_to = (uint8_t *)to->d_k_block_scales;
        e.v_blocks_to = (uint8_t *)to->d_v_block_scales;
    }
    LAUNCH_TRY(zc::launch_evict(e, stream));
    return ZC_OK;
}
