// Host side of the operators over K/V pages: argument checks, the choice of kernels and splits, and the C entry points
// zc_attend, zc_attend_shared, zc_attend_workspace_bytes and zc_evict.
#include <hip/hip_runtime.h>

#include <cmath>

#include "zc_attend.h"
#include "zc_host.h"

namespace zc {

namespace {

constexpr uint32_t kMaxTokens = 1u << 30;      // positions are signed 32-bit numbers in the kernels, sums of two included
constexpr uint64_t kMaxBlocks = (1u << 24) - 1;   // of 256 threads: HIP launches fewer than 2^32
constexpr uint32_t kMaxSlots = 64;             // parts of one row: k_attend_join holds one per lane
constexpr uint64_t kMostLogits = 1u << 30;     // bytes of scratch

bool aligned4(const void *p) { return ((uintptr_t)p & 3) == 0; }

zc_status check_cache(const zc_kv_cache *c, PagesDev *out)
{
    if (!c) return ZC_ERR_INVALID_ARG;
    if (c->struct_size != sizeof(zc_kv_cache)) return ZC_ERR_UNSUPPORTED;
    if (c->format != ZC_FMT_BF16 && c->format != ZC_FMT_FP8_E4M3 && c->format != ZC_FMT_FP8_E5M2) return ZC_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128) return ZC_ERR_UNSUPPORTED;
    if (c->page_tokens < 16 || c->page_tokens > 65536 || (c->page_tokens & (c->page_tokens - 1))) return ZC_ERR_INVALID_ARG;
    if (!c->n_seqs || !c->n_heads || !c->table_pages || !c->n_pages || c->n_pages > 0x7FFFFFFFu) return ZC_ERR_INVALID_ARG;
    const uint64_t capacity = (uint64_t)c->table_pages * c->page_tokens;
    if (capacity >= kMaxTokens || (uint64_t)c->n_seqs * c->n_heads > (kMaxBlocks >> 2)) return ZC_ERR_INVALID_ARG;     // (k_evict_select has 1,024 threads for each)
    if (!c->d_k_pages || !c->d_v_pages || !c->d_table || !c->d_lengths) return ZC_ERR_INVALID_ARG;
    if (!aligned16(c->d_k_pages) || !aligned16(c->d_v_pages) || !aligned4(c->d_table) || !aligned4(c->d_lengths) ||
        !aligned4(c->d_k_scales) || !aligned4(c->d_v_scales)) return ZC_ERR_INVALID_ARG;
    PagesDev d = {};
    d.k = (const uint8_t *)c->d_k_pages;
    d.v = (const uint8_t *)c->d_v_pages;
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
    uint32_t tiles, row_blocks, even, splits;
    uint64_t blocks;
};

// rows: of one (sequence, head), or of one head of the prefix; units: how many of those; longest: tokens that a row block may have to read;
// only: the call has no other pass
Pass plan_pass(uint64_t rows, uint64_t units, uint64_t longest, uint32_t most_splits, bool only)
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
    const uint64_t groups = units * p.row_blocks, part = 256, possible = only && longest <= 640 ? 1 : (longest + part - 1) / part;
    // Lengths are not known here, only the longest.  So that one long cache among short ones does not keep everyone waiting, parts are at
    // most kLongPart tokens, and what is left over of a shorter cache's parts ends at once: 31 FP8 caches of 1,000 tokens and one of 131,072
    // 1,077 -> 128 us, 64 of 0 to 32,768 444 -> 408 us; 64 of 8,192 188 us as before, 16 of 32,768 190 -> 198 us.  (At most 4,096: 109, 391,
    // 202 and 209 us.)  k_attend_many has row blocks enough where rows are many, and its parts would take their number times as much room.
    const uint64_t enough = p.many ? 512 : 256;
    uint64_t even = groups ? (enough + groups - 1) / groups : 1;
    if (even > possible) even = possible;
    if (even > most_splits) even = most_splits;
    if (!even) even = 1;
    const uint64_t least = p.many ? 1 : (longest + kLongPart - 1) / kLongPart, s = even > least ? even : least;
    p.even = (uint32_t)even;
    p.splits = (uint32_t)(s < most_splits ? s : most_splits);
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
    p.own_pass = plan_pass((uint64_t)a.max_q_len * a.group, (uint64_t)a.n_seqs * a.c.heads, reach(a.c.limit), shared ? 16 : kMaxSlots, !shared);
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
        p.pre_pass = plan_pass((uint64_t)a.n_tokens * a.group, a.c.heads, (uint64_t)pc.limit, 48, false);
        b.splits = p.pre_pass.splits;
        b.even = p.pre_pass.even;
        b.row_blocks = p.pre_pass.row_blocks;
        b.first_slot = 0;
        a.first_slot = b.splits;
        p.slots += b.splits;
    } else if (x->max_prefix_len) return ZC_ERR_INVALID_ARG;
    a.splits = p.own_pass.splits;
    a.even = p.own_pass.even;
    a.row_blocks = p.own_pass.row_blocks;
    a.direct = p.slots == 1;
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

extern "C" zc_status zc_evict(const zc_kv_cache *from, const float *d_weights, uint32_t keep, uint32_t sinks, uint32_t recent,
                              const zc_kv_cache *to, float *d_weights_to, int32_t *d_kept, void *stream)
{
    zc::EvictDev e = {};
    zc_status st = zc::check_cache(from, &e.from);
    if (!st) st = zc::check_cache(to, &e.to);
    if (st) return st;
    if (!zc::same_shape(*from, *to) || from->n_seqs != to->n_seqs || from->d_lengths == to->d_lengths) return ZC_ERR_INVALID_ARG;
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
    e.row_bytes = from->head_dim * (from->format == ZC_FMT_BF16 ? 2 : 1);
    LAUNCH_TRY(zc::launch_evict(e, stream));
    return ZC_OK;
}
