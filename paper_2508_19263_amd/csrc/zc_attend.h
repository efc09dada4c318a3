// Internal declarations of the operators over K/V pages (zc_attend*, zc_evict): what the host side (zc_attend.cpp) hands to
// the kernels (zc_attend_*.hip, zc_evict.hip).  Not part of the C ABI.
#pragma once
#include <stdint.h>

#include "../../include/zc.h"

namespace zc {

// A paged cache as the kernels see it: `page_shift` is the logarithm of page_tokens, `capacity` the tokens a table has room for.
struct PagesDev {
    const uint8_t *k, *v;
    const int32_t *table;              // [seqs][heads][table_pages]
    const int32_t *lengths;            // [seqs]
    const float *k_scales, *v_scales;  // [seqs][heads] or null
    const uint8_t *k_blocks, *v_blocks;        // FP4: block scales of the pages' rows
    uint32_t heads, table_pages, n_pages, page_shift;
    int32_t capacity, limit;           // longer lengths are taken as `limit`
};

// One pass of attention over one cache: query rows against the tokens of `c`, split into `splits` parts.
struct AttendDev {
    PagesDev c;
    const uint16_t *q;
    uint16_t *out;
    float *lse;                        // [tokens][q heads] or null
    const int32_t *q_start;            // [seqs + 1] or null: one token per sequence
    const int32_t *own_lengths;        // lengths of the sequences' own caches: they give the positions
    const int32_t *prefix_length;      // length of the shared prefix or null
    float *part_o, *part_ml;           // workspace: [slot][row][dim] and [slot][row][2], rows in the order of lse
    uint64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;   // elements
    float *logits;                     // k_attend_few with at most kLogitRows rows, or null: [seq][head][logit_rows][logit_stride], in base 2
    uint32_t logit_rows, logit_stride;
    float scale;
    int32_t own_limit, prefix_limit;
    uint32_t n_seqs, n_tokens, q_heads, group, max_q_len, window, sinks;
    uint32_t shared;                   // 1: `c` is the prefix, and a row block takes rows of all sequences
    uint32_t splits, first_slot;       // this pass's slots are first_slot .. first_slot + splits
    uint32_t even, long_part;          // k_attend_few: parts that what a sequence sees is divided into if these have no more than so many tokens
    uint32_t row_blocks;               // row blocks per (sequence, head), or per head of the prefix
    uint32_t past_caches;              // k_attend_few: tokens of all sequences above which pages go past the caches; 0: none do
    int32_t reach;                     // tokens of a sequence that are read, at most
    uint32_t eight;                    // 1: k_attend_short in k_attend_few's place
    uint32_t direct;                   // 1: one slot in all, the pass writes out and lse itself
};

constexpr uint64_t kMemorySideCache = 256u << 20;     // bytes
constexpr uint32_t kLeastPast = 64;    // bytes of a row that may go past them
constexpr int32_t kLeastChoice = 768;  // tokens of a part that is worth choosing for
constexpr uint32_t kMostParts = 16;
constexpr uint32_t kLogitRows = 24;    // rows whose logits k_attend_few leaves
constexpr uint32_t kLongPart = 8192;   // tokens; of FP4 half of it, or
constexpr uint32_t kShortPart = 2560;

struct WeightsDev {
    const float *in;                   // or null
    float *out;                        // [seqs][heads][capacity]
    float *part;                       // workspace: [parts][seqs][heads][limit] where parts > 1
    uint32_t parts;                    // workgroups of k_attend_weights that share tokens, at most kMostParts
};

struct EvictDev {
    PagesDev from, to;
    uint8_t *k_to, *v_to;
    const float *weights;              // [seqs][heads][from.capacity]
    float *weights_to;                 // [seqs][heads][to.capacity] or null
    int32_t *kept;                     // [seqs][heads][keep]
    int32_t *lengths_to;
    uint8_t *k_blocks_to, *v_blocks_to;
    uint32_t n_seqs, keep, sinks, recent, row_bytes;
    uint32_t row_scales;               // FP4: bytes of a row's block scales; else 0
};

// Rows of the last tokens of sequences, to be written to a cache or read back from it.
struct RowsDev {
    PagesDev c;
    uint8_t *k_pages, *v_pages, *k_scale_pages, *v_scale_pages;       // what is written to
    uint16_t *k, *v;                   // BF16 [tokens][heads][dim]
    uint64_t k_token_stride, k_head_stride, v_token_stride, v_head_stride;       // elements
    const int32_t *q_start;            // [seqs + 1] or null: one token per sequence
    uint32_t n_seqs, n_tokens;
};

// tiles: of 16 rows in k_attend_few, of 128 in k_attend_many
int launch_attend_few(const AttendDev &a, uint32_t format, uint32_t head_dim, uint32_t tiles, void *stream);
int launch_attend_many(const AttendDev &a, uint32_t format, uint32_t head_dim, void *stream);
// both passes of a shared prefix; tiles: of 16 rows, of the own pass and of the prefix where that is not pre_many
int launch_attend_shared(const AttendDev &pre, const AttendDev &own, uint32_t format, uint32_t head_dim, bool pre_many, uint32_t tiles, void *stream);
// slots > 1: joins them; a.logits: adds up the weights from them
int launch_attend_join(const AttendDev &a, const WeightsDev &w, uint32_t head_dim, uint32_t slots, void *stream);
int launch_attend_weights(const AttendDev &a, const WeightsDev &w, uint32_t format, uint32_t head_dim, void *stream);
int launch_evict(const EvictDev &e, void *stream);
int launch_kv_write(const RowsDev &r, uint32_t format, uint32_t head_dim, void *stream);
int launch_kv_read(const RowsDev &r, uint32_t format, uint32_t head_dim, void *stream);

}  // namespace zc
