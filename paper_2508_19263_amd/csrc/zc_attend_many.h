// Attention over K/V pages for many query rows (prompts, batches under one prefix): the body of k_attend_many, and of
// the part of k_attend_shared that is like it.
//
// A workgroup of four wavefronts takes 128 rows of one K/V head, 32 to a wavefront, and goes over the tokens
// they see 64 at a time.  A tile of keys and values is brought to LDS once for all of them, in the type it is multiplied in (BF16 goes
// there past the registers; FP8 is converted on the way: keys to BF16, values to half precision), into one of two buffers while the
// other is worked on:
//   S^T = K Q^T     32 tokens x 32 rows per instruction; a lane holds one row's products with half of the tile's tokens
//   O^T += V^T P^T  a lane's weights are its operand as they stand; V comes from LDS through transposing reads, four tokens
//                   of a dimension at a time, which are exactly the runs of four tokens that S^T leaves in a lane
// The bank a 16-byte piece of a key (64-byte piece of a value) lies in depends on its token too, so that neither the reads of
// 16 tokens' pieces nor the transposing ones meet in a bank.
//
// Measured with 8 K/V heads of 128 and 4 query heads to each: two BF16 prompts of 8,192 and 7,001 tokens with a window of 4,096 and 16
// sinks 790 - 850 us, 880 - 945 TFLOP/s (counted are the products of tokens that are seen); pieces of 1,024 and 511 tokens behind 7,977
// and 7,680 FP8 ones 137 - 147 us, 700 - 750 TFLOP/s.  A library product of 8,192^3 reaches 1,136 on this card, and its clock goes down to 1.5 GHz
// under it; here it goes from 2.2 to 1.9.  The matrix unit is busy 51 % of the cycles (FP8: 38 %), the exponentials and what belongs to
// them take about as many (two wavefronts to a SIMD; registers and LDS have room for no more); other orders of the same instructions
// give the same time.
#pragma once
#include "zc_attend_device.h"

namespace zc {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr uint32_t kManyWaves = 4;
constexpr int kTile = 64;                      // tokens per step
constexpr int kSchedMatrix = 0x8, kSchedLdsRead = 0x100, kReadsAhead = 6;   // kinds of instructions for __builtin_amdgcn_sched_group_barrier
constexpr int kHalves = kTile / 32, kStretches = kTile / 16;

template <int FMT> __device__ __forceinline__ f32x16 mma32_values(u32x4_t a, u32x4_t b, f32x16 c)
{
    if constexpr (FMT == ZC_FMT_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
}
template <int FMT> __device__ __forceinline__ u32x4_t eight_to_half(uint32_t lo, uint32_t hi)
{
    return u32x4_t{two_to_half<FMT, false>(lo), two_to_half<FMT, true>(lo), two_to_half<FMT, false>(hi), two_to_half<FMT, true>(hi)};
}

// Byte offset in a tile of 64 tokens x D two-byte elements of values: byte x of a token's row, moved in pieces of 64 bytes.
template <int D> __device__ __forceinline__ uint32_t value_place(uint32_t token, uint32_t x)
{
    return D == 128 ? token * 256 + (x ^ ((token & 3) << 6)) : token * 128 + (x ^ ((token >> 1 & 1) << 6));
}

// A workgroup's LDS.  The two buffers are variables of their own, so that the compiler knows what is brought to one of them does not
// lie in the other, and reads of the other need not wait for it.
template <int D> struct ManyTile {
    alignas(1024) uint8_t keys[kTile * D * 2], values[kTile * D * 2];
};
struct ManyNotes {
    uint32_t bad_tokens[3][kHalves];                           // [tile modulo 3]: tokens with an element that is not finite
    int32_t limits[kManyWaves][4];
};

// 16 bytes at a lane's own offset to the lane's place in a wavefront's 1,024 consecutive bytes of LDS
__device__ __forceinline__ void bring(__amdgpu_buffer_rsrc_t from, uint32_t at, uint8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, (int)at, 0, 0, 0);
}
__device__ __forceinline__ void wait_for_brought() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <int FMT, int D>
__device__ __forceinline__ void attend_many(const AttendDev &a, uint32_t id, ManyTile<D> &tile0, ManyTile<D> &tile1, ManyNotes &notes)
{
    constexpr bool kBring = FMT == ZC_FMT_BF16;                // tiles go to LDS as they are, past the registers
    constexpr int ES = PageElem<FMT>::BYTES, KS = D / 16, DT = D / 32;
    constexpr uint32_t kPieces = D * ES / 16;                  // 16-byte pieces of a stored row
    constexpr uint32_t kRowsPerPass = 64 / kPieces, kPasses = 16 / kRowsPerPass;
    auto &bad_tokens = notes.bad_tokens;
    auto &limits = notes.limits;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n32 = lane & 31, g = lane >> 5;
    const uint32_t units = (a.shared ? 1 : a.n_seqs) * a.c.heads;
    const uint32_t unit = id % units;                          // neighbours on an XCD work on the same few heads
    id /= units;
    const uint32_t split = id % a.splits, row_block = a.row_blocks - 1 - id / a.splits;    // the long rows of a prompt first
    const uint32_t head = unit % a.c.heads, seq = unit / a.c.heads;

    const int32_t prefix = prefix_tokens(a), offset = a.shared ? 0 : prefix;
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit);
    const Span span = rows_span(a, seq);
    const uint32_t first_row = row_block * (kManyWaves * 32);
    if ((uint64_t)first_row >= (uint64_t)span.count * a.group) return;         // the whole workgroup
    const Row row = row_of(a, span, head, first_row + wave * 32 + n32, prefix, offset, length);
    int32_t last_min = INT32_MAX, last_max = -1, from_min = INT32_MAX, from_max = INT32_MIN;
    if (row.token >= 0) {
        last_min = last_max = row.sight.last;
        from_min = from_max = row.sight.from;
    }
    last_min = min_over_wave(last_min);
    last_max = max_over_wave(last_max);
    from_min = min_over_wave(from_min);
    from_max = max_over_wave(from_max);
    if (lane == 0) { limits[wave][0] = last_min; limits[wave][1] = last_max; limits[wave][2] = from_min; limits[wave][3] = from_max; }
    if (tid < 3 * kHalves) (&bad_tokens[0][0])[tid] = 0;
    __syncthreads();
    // the same of the whole workgroup
    int32_t all_last_min = INT32_MAX, all_last_max = -1, all_from_min = INT32_MAX, all_from_max = INT32_MIN;
    for (uint32_t w = 0; w < kManyWaves; w++) {
        all_last_min = min(all_last_min, uniform(limits[w][0]));
        all_last_max = max(all_last_max, uniform(limits[w][1]));
        all_from_min = min(all_from_min, uniform(limits[w][2]));
        all_from_max = max(all_from_max, uniform(limits[w][3]));
    }
    const int32_t sinks = (int32_t)a.sinks - offset;
    const Blocks blocks = seen_blocks(kTile, all_last_max, all_from_min, sinks);
    const int32_t per_split = (blocks.count + (int32_t)a.splits - 1) / (int32_t)a.splits;
    const int32_t begin = min((int32_t)split * per_split, blocks.count), end = min(begin + per_split, blocks.count);

    const float k_scale = a.c.k_scales ? a.c.k_scales[unit] : 1.0f, v_scale = a.c.v_scales ? a.c.v_scales[unit] : 1.0f;
    const float signed_c = a.scale * k_scale * kLog2e;
    // logits in base 2 (for signs and NaN see query_operand)
    const float c = fmaxf(fabsf(signed_c), kLeastFactor);
    u32x4_t q[KS];
    {
        const uint16_t *from = a.q + (uint64_t)max(row.token, 0) * a.q_token_stride + (uint64_t)row.q_head * a.q_head_stride;
#pragma unroll
        for (int u = 0; u < KS; u++) {
            u32x4_t x = {0, 0, 0, 0};
            if (row.token >= 0) x = *reinterpret_cast<const u32x4_t *>(from + u * 16 + g * 8);
            q[u] = query_operand(x, signed_c);
        }
    }
    float base = kNoBase, l = 0.0f;                            // what the row's logits are taken relative to; sum over this lane's tokens
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[d][i] = 0.0f;

    // ---- bringing tiles: a wavefront takes 16 tokens, which lie in one page, some rows at a time; a lane has piece `piece` of each
    const int32_t *table = a.c.table + (uint64_t)unit * a.c.table_pages;
    const uint32_t page_log = a.c.page_shift + (D == 128 ? 7 : 6) + (ES - 1);   // of a page's bytes
    const uint32_t page_mask = (1u << a.c.page_shift) - 1;
    const uint32_t piece = lane % kPieces, row0 = wave * 16 + lane / kPieces;       // (the row of pass 0)
    // lane kStretches * i + h: page of tokens 16 h .. of tile ids_from + i (0 where it is absent), and the bit that says it is there
    int32_t ids = 0, ids_from = begin;
    uint64_t present = 0;
    auto fetch_ids = [&](int32_t b) {
        const int32_t mine = b + (int32_t)(lane / kStretches);
        const uint32_t page = ((uint32_t)blocks.at(mine) * kTile + (lane % kStretches) * 16) >> a.c.page_shift;
        int32_t id = -1;
        if (mine < end && page < a.c.table_pages) id = table[page];
        const bool there = (uint32_t)id < a.c.n_pages;
        present = __ballot(there);
        ids = there ? id : 0;
        ids_from = b;
    };
    // which of a tile's stretches of 16 tokens are present
    auto there_of = [&](int32_t b) { return (uint32_t)(present >> ((b - ids_from) * kStretches)) & ((1u << kStretches) - 1); };
    u32x4_t kx[kPasses], vx[kPasses];
    // Where a lane's piece of a pass lies from the first of the 16 tokens.  kBring: place `piece` of a row of LDS holds another piece of
    // it, by key_place and value_place, whose exchange of pieces is its own inverse.
    auto mine_k = [&](uint32_t p) {
        const uint32_t r = row0 + p * kRowsPerPass;
        return (r & 15) * (D * ES) + (kBring ? key_place<D>(r, piece) & (D * 2 - 1) : piece * 16);
    };
    auto mine_v = [&](uint32_t p) {
        const uint32_t r = row0 + p * kRowsPerPass;
        return (r & 15) * (D * ES) + (kBring ? value_place<D>(r, piece * 16) & (D * 2 - 1) : piece * 16);
    };
    auto fetch = [&](int32_t b, ManyTile<D> &to) {
        const uint32_t t0 = (uint32_t)blocks.at(b) * kTile + wave * 16, page = (uint32_t)__builtin_amdgcn_readlane(ids, (b - ids_from) * kStretches + (int32_t)wave);
        const uint64_t where = ((uint64_t)page << page_log) + (t0 & page_mask) * (D * ES);
        const __amdgpu_buffer_rsrc_t k = sixteen_tokens(a.c.k + where, 16 * D * ES), v = sixteen_tokens(a.c.v + where, 16 * D * ES);
#pragma unroll
        for (uint32_t p = 0; p < kPasses; p++) {
            if constexpr (kBring) {
                bring(k, mine_k(p), to.keys + wave * (16 * D * 2) + p * 1024);
                bring(v, mine_v(p), to.values + wave * (16 * D * 2) + p * 1024);
            } else {
                kx[p] = __builtin_amdgcn_raw_buffer_load_b128(k, (int)mine_k(p), 0, 0);
                vx[p] = __builtin_amdgcn_raw_buffer_load_b128(v, (int)mine_v(p), 0, 0);
            }
        }
    };
    // whether every row of the workgroup (of the wavefront) sees every token of a tile
    auto whole = [&](int32_t t0, uint32_t there, int32_t lmin, int32_t fmax) { return there == (1u << kStretches) - 1 && t0 + kTile - 1 <= lmin && (t0 >= fmax || t0 + kTile <= sinks); };
    auto store_keys = [&](ManyTile<D> &to) {
        if constexpr (!kBring) {
#pragma unroll
            for (uint32_t p = 0; p < kPasses; p++) {
                const uint32_t r = p * kRowsPerPass + row0;
                *reinterpret_cast<u32x4_t *>(to.keys + key_place<D>(r, piece * 2)) = eight_to_bf16<FMT>(kx[p][0], kx[p][1]);
                *reinterpret_cast<u32x4_t *>(to.keys + key_place<D>(r, piece * 2 + 1)) = eight_to_bf16<FMT>(kx[p][2], kx[p][3]);
            }
        }
    };
    // Tokens that no row sees are zeroed (what they hold is not to be multiplied, not even with 0); of those that only some rows see,
    // elements that are not finite are zeroed too and noted: they are added to the rows that do see them.
    auto clean = [&](u32x4_t &x, uint32_t r, int32_t t0, uint32_t there, uint32_t mod3) {
        const int32_t t = t0 + (int32_t)r;
        const bool used = (there >> wave & 1) && seen(Sight{all_last_max, all_from_min, sinks}, t);
        const bool by_all = seen(Sight{all_last_min, all_from_max, sinks}, t);
        uint32_t wild = 0;
#pragma unroll
        for (int w = 0; w < 4; w++) {
            x[w] = used ? x[w] : 0u;
            const uint32_t y = by_all ? 0u : nonfinite_mask<FMT>(x[w]);
            wild |= y;
            x[w] &= ~y;
        }
        if (wild) atomicOr(&bad_tokens[mod3][r / 32], 1u << (r & 31));
    };
    auto store_values = [&](int32_t t0, uint32_t there, bool edge, ManyTile<D> &to, uint32_t mod3) {
        if constexpr (kBring) {
            wait_for_brought();
            if (__builtin_expect(edge, 0)) {
#pragma unroll
                for (uint32_t p = 0; p < kPasses; p++) {
                    u32x4_t *place = reinterpret_cast<u32x4_t *>(to.values + wave * (16 * D * 2) + p * 1024 + lane * 16);
                    u32x4_t x = *place;
                    clean(x, p * kRowsPerPass + row0, t0, there, mod3);
                    *place = x;
                }
            }
        } else {
            if (__builtin_expect(edge, 0)) {
#pragma unroll
                for (uint32_t p = 0; p < kPasses; p++) clean(vx[p], p * kRowsPerPass + row0, t0, there, mod3);
            }
#pragma unroll
            for (uint32_t p = 0; p < kPasses; p++) {
                const uint32_t r = p * kRowsPerPass + row0;
                *reinterpret_cast<u32x4_t *>(to.values + value_place<D>(r, piece * 32)) = eight_to_half<FMT>(vx[p][0], vx[p][1]);
                *reinterpret_cast<u32x4_t *>(to.values + value_place<D>(r, piece * 32 + 16)) = eight_to_half<FMT>(vx[p][2], vx[p][3]);
            }
        }
    };

    // Product 16 h + i of a tile is the lane's row with token 32 h + (i / 4) * 8 + g * 4 + i % 4.
    struct Products { f32x16 half[kHalves]; };
    // one of the steps of S^T = K Q^T: 16 dimensions
    auto multiply_keys = [&](const uint8_t *kt, int u, Products &s) {
#pragma unroll
        for (int h = 0; h < kHalves; h++) {
            const u32x4_t key = *reinterpret_cast<const u32x4_t *>(kt + key_place<D>(h * 32 + n32, u * 2 + g));
            const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
            s.half[h] = mma32_keys(key, q[u], u ? s.half[h] : zero);
        }
    };
    auto hide = [&](int32_t t0, uint32_t there, Products &s) {      // what the row does not see
        if (__builtin_expect(!whole(t0, there, last_min, from_max), 0)) {
            uint32_t mask = 0;
#pragma unroll
            for (int n = 0; n < kTile / 8; n++) mask |= (seen_of_four(row.sight, t0 + n * 8 + (int32_t)g * 4) & (there >> (n / 2) & 1 ? 15u : 0u)) << (n * 4);
#pragma unroll
            for (int i = 0; i < kTile / 2; i++) {
                const uint32_t keep = bit_as_mask(mask, i);
                s.half[i / 16][i & 15] = __uint_as_float((bits(s.half[i / 16][i & 15]) & keep) | (bits(kNegInf) & ~keep));
            }
        }
    };
    auto top_of = [&](const Products &s) {
        float top = s.half[0][0];
#pragma unroll
        for (int i = 1; i < kTile / 2; i++) top = fmaxf(top, s.half[i / 16][i & 15]);
        return max_over_32(top);
    };
    auto raise = [&](float top) {                              // the base, where a product has left it far behind
        if (__builtin_expect(__any(out_of_reach<FMT>(base, top, c)), 0)) {
            const float now = raised<FMT>(base, top, c);
            const float f = __builtin_amdgcn_exp2f(base - now);
            base = now;
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; d++) o[d] *= f;
        }
    };

    auto multiply = [&](const ManyTile<D> &tile, Products &s) {
        const uint8_t *kt = tile.keys;
        // Of the two wavefronts of a SIMD the one at its matrix instructions goes first, and the other one's arithmetic fills in: two
        // prompts 885 -> 870 us, pieces of prompts 158 -> 149 us (the other way round 898 and 162 us).
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int u = 0; u < KS; u++) multiply_keys(kt, u, s);
        // reads of keys run ahead of their products
        __builtin_amdgcn_sched_group_barrier(kSchedLdsRead, kReadsAhead, 0);
#pragma unroll
        for (int i = 0; i < 2 * KS; i++) {
            __builtin_amdgcn_sched_group_barrier(kSchedMatrix, 1, 0);
            if (i + kReadsAhead < 2 * KS) __builtin_amdgcn_sched_group_barrier(kSchedLdsRead, 1, 0);
        }
    };
    auto rest = [&](int32_t t0, uint32_t there, bool edge, const ManyTile<D> &tile, uint32_t mod3, Products &s) {
        const uint8_t *vt = tile.values;
        if (__builtin_expect(edge, 0)) hide(t0, there, s);
        raise(top_of(s));
        float sum[4] = {0, 0, 0, 0};
        u32x4_t p[kStretches];
#pragma unroll
        for (int i = 0; i < kTile / 2; i++) {
            const float e = weight_of(s.half[i / 16][i & 15], c, base);                       // (0 for the products hidden above)
            s.half[i / 16][i & 15] = e;
            sum[i & 3] += e;
            if (i & 1) p[i / 8][i / 2 & 3] = pack_weights<FMT>(s.half[i / 16][(i & 15) - 1], e);
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        uint64_t bad = 0;
        if (__builtin_expect(edge, 0)) bad = (uint64_t)uniform(bad_tokens[mod3][0]) | (uint64_t)uniform(bad_tokens[mod3][1]) << 32;
        if (__builtin_expect(bad != 0, 0)) {
#pragma unroll 1
            for (uint32_t n = 0; n < kTile; n++) {
                if (!(bad >> n & 1)) continue;
                const uint32_t i = (n >> 5) * 16 + (n & 3) + (n >> 3 & 3) * 4, gg = n >> 2 & 1;        // product i, in the lanes of group gg
                uint32_t word = p[0][0];
#pragma unroll
                for (uint32_t k = 1; k < kTile / 4; k++) word = i / 2 == k ? p[k / 4][k & 3] : word;
                word = (uint32_t)__shfl((int)word, (int)(n32 + gg * 32)) >> (i & 1) * 16 & 0xFFFFu;
                const float weight = FMT == ZC_FMT_BF16 ? __uint_as_float(word << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)word);
                const int32_t tok = t0 + (int32_t)n;
                const bool mine = seen(row.sight, tok);
                const uint8_t *from = a.c.v + ((uint64_t)(uint32_t)max(table[(uint32_t)tok >> a.c.page_shift], 0) << page_log) + ((uint32_t)tok & page_mask) * (D * ES);
#pragma unroll
                for (int d = 0; d < DT; d++)
#pragma unroll
                    for (int kk = 0; kk < 16; kk += 4) {
#pragma unroll
                        for (int k = kk; k < kk + 4; k++) {
                            const float x = element<FMT>(from + (d * 32 + (k / 4) * 8 + (int)g * 4 + (k & 3)) * ES);
                            o[d][k] += mine && !(fabsf(x) < __builtin_inff()) ? weight * x : 0.0f;
                        }
                        __builtin_amdgcn_sched_barrier(0);       // a few at a time: this hardly ever runs and is to cost no registers
                    }
            }
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < kStretches; k++)
#pragma unroll
            for (int d = 0; d < DT; d++) {
                // lanes of a group of 16: four tokens, four 8-byte pieces of 16 dimensions
                const uint32_t tok = k * 16 + g * 4 + (lane >> 2 & 3), x = d * 64 + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
                const u32x2 lw = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + value_place<D>(tok, x))));
                const u32x2 hw = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + value_place<D>(tok + 8, x))));
                o[d] = mma32_values<FMT>(u32x4_t{lw[0], lw[1], hw[0], hw[1]}, p[k], o[d]);
            }
    };

    // Two buffers.  The next tile goes straight to the other buffer while a tile is worked on (BF16: two prompts of 8,192 and 7,001 tokens
    // 916 -> 847 us against the way through registers), or, where it is converted, is asked for when the tile's products have been made,
    // waits in registers while their weights are worked out and the values multiplied, and is stored then.  (Asked for a whole step ahead, it
    // takes the registers that reading keys ahead needs.  So does making a tile's products beside the exponentials of the one before
    // it, in 32 or 64 tokens: 6 to 12 % slower.)
    if (begin < end) {
        fetch_ids(begin);
        uint32_t there = there_of(begin), mod3 = 0;
        int32_t t0 = blocks.at(begin) * kTile;
        bool edge = !whole(t0, there, all_last_min, all_from_max);             // some row of the workgroup does not see all of the tile
        fetch(begin, tile0);
        store_keys(tile0);
        store_values(t0, there, edge, tile0, 0);
        __syncthreads();
        auto step = [&](int32_t b, ManyTile<D> &tile, ManyTile<D> &next) {
            const uint32_t next3 = mod3 == 2 ? 0 : mod3 + 1;
            const int32_t later = min(b + 1, end - 1);                         // (the last one is asked for again: no branch, no wait)
            const bool ours = t0 <= last_max && (t0 + kTile > from_min || t0 < sinks);  // else nothing of the tile is for this wavefront's rows
            if (later - ids_from >= 64 / kStretches) fetch_ids(later);
            const uint32_t there_next = there_of(later);
            const int32_t t0_next = blocks.at(later) * kTile;
            const bool edge_next = !whole(t0_next, there_next, all_last_min, all_from_max);
            Products s;
            if constexpr (kBring) fetch(later, next);
            if (ours) multiply(tile, s);
            __builtin_amdgcn_s_setprio(0);
            if constexpr (!kBring) fetch(later, next);
            if (ours) rest(t0, there, edge, tile, mod3, s);
            __builtin_amdgcn_s_setprio(0);
            store_keys(next);
            store_values(t0_next, there_next, edge_next, next, next3);
            if (tid < kHalves) bad_tokens[next3 == 2 ? 0 : next3 + 1][tid] = 0;        // last read before the barrier that began this step
            there = there_next;
            t0 = t0_next;
            edge = edge_next;
            __syncthreads();
            mod3 = next3;
        };
        for (int32_t b = begin; b < end; b += 2) {
            step(b, tile0, tile1);
            if (b + 1 < end) step(b + 1, tile1, tile0);
        }
    }

    // ---- results: a lane has 4 consecutive dimensions at a time
    if (row.token < 0) return;
    const float sum = sum_over_32(l);
    const float top = part_base(base, sum);
    const uint64_t at = (uint64_t)row.token * a.q_heads + row.q_head;
    if (a.direct) {
        const float inv = sum == 0.0f ? 0.0f : v_scale / sum;
        uint16_t *to = a.out + (uint64_t)row.token * a.out_token_stride + (uint64_t)row.q_head * a.out_head_stride + g * 4;
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const u32x2 w = {pack_bf16(o[d][k * 4] * inv, o[d][k * 4 + 1] * inv), pack_bf16(o[d][k * 4 + 2] * inv, o[d][k * 4 + 3] * inv)};
                *reinterpret_cast<u32x2 *>(to + d * 32 + k * 8) = w;
            }
        if (a.lse && g == 0) a.lse[at] = sum == 0.0f ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    } else {
        const uint64_t slot = (uint64_t)(a.first_slot + split) * a.n_tokens * a.q_heads + at;
        float *to = a.part_o + slot * D + g * 4;
        if (begin < end)                                       // (else k_attend_join does not look at it)
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
            for (int k = 0; k < 4; k++)
                *reinterpret_cast<f32x4 *>(to + d * 32 + k * 8) = f32x4{o[d][k * 4] * v_scale, o[d][k * 4 + 1] * v_scale, o[d][k * 4 + 2] * v_scale, o[d][k * 4 + 3] * v_scale};
        if (g == 0) { a.part_ml[slot * 2] = top; a.part_ml[slot * 2 + 1] = sum; }
    }
}

}  // namespace zc
