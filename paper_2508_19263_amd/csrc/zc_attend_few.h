// Attention over K/V pages for few query rows (decoding): the body of k_attend_few, and of the part of k_attend_shared that is like it.
//
// The rows of one (sequence, K/V head), its query tokens times the query heads that share the K/V head, are few, and the
// cache is long: the kernel is bound by the read of the pages.  Each wavefront takes every fourth block of 32 tokens of its
// workgroup's part of the cache and multiplies it with all rows, 16 at a time, straight from registers:
//   S^T = K Q^T      a lane holds one query row's products with 2 x 4 tokens; the base they are taken relative to and their sum l go with it
//   O^T += V^T P^T   those 8 weights are the lane's operand as they stand: the order of the tokens in the sum is free, so the
//                    lane that holds rows of V for the product takes those of the same 8 tokens
// Neither K, V nor the weights pass through LDS; V is transposed by byte permutes inside a lane, which holds 8 tokens x
// head_dim / 16 consecutive dimensions.  At the end the wavefronts' (m, l, O) are joined in LDS; parts of a cache that went
// to different workgroups are joined by k_attend_join.
//
// Measured with 8 K/V heads of 128 in random pages of 16 tokens, one query token, 4 query heads to each, joins included (a large element-wise
// pass reaches 6.2 TB/s): 64 FP8 caches of 8,192 tokens 167 us, 6.4 TB/s (past the caches; 212 where their memory lies less well, which no address
// tells); 48 BF16 ones of 12,000 373 - 420 us, 5.6 - 6.3 TB/s; 4 FP8 ones of 8,192 16.5 us, 4.1 TB/s; one with 512 tokens in sight 8.5 us, all latency.
//
// FP4 elements are converted as they are used, with their block's scale: MX to BF16, an instruction for two keys, two for two values (the tokens
// have to be paired); NV keys to BF16 (four instructions), values to half precision (two and a quarter).  64 MXFP4 caches of 8,192 tokens
// 103 us, 5.5 TB/s of what they hold: the read, and 200 vector instructions for 32 tokens, which take 53 % of the time beside it; NVFP4 120 us,
// 5.0 TB/s, 340 instructions, which take 62 %.  (NV keys and queries in half precision, where queries have to be brought to its range and rows that
// do not fit it need a loop of their own, are 80 instructions less: 32 caches of 16,384 125.4 -> 128.6 us, shorter ones the same.  A step
// more ahead, in two sets of registers: MX 113 -> 120, NV 126 -> 130.)
#pragma once
#include "zc_attend_device.h"

namespace zc {

constexpr uint32_t kWaves = 4;                 // wavefronts per workgroup (k_attend_few: with eight, batches were 1 us slower and single sequences 0.6 us faster: see k_attend_short)

template <int FMT, int D> struct BlockRegs {
    static constexpr int NK = D * kElemBits<FMT> / 512;              // 16-byte pieces of a key per lane
    static constexpr int DL = D / 16, VW = DL * kElemBits<FMT> / 32; // dimensions and words of a value per lane
    u32x4_t k[2][NK];
    uint32_t v[8][VW];
};
// FP4: a quarter of a key, in words of eight elements, and its one or two block scales; D / 16 consecutive dimensions (a word or half of one) of
// a value and their block's scale.
template <int FMT, int D> struct BlockRegs4 {
    static constexpr int DL = D / 16, KW = D / 32;
    uint32_t k[2][KW], k_scale[2];
    uint32_t v[8], v_scale[8];
};
template <int FMT, int D, bool FP4 = kFp4<FMT>> struct FewRegs { typedef BlockRegs<FMT, D> Type; };
template <int FMT, int D> struct FewRegs<FMT, D, true> { typedef BlockRegs4<FMT, D> Type; };

template <int AUX, int N> __device__ __forceinline__ void load_words(uint32_t (&to)[N], __amdgpu_buffer_rsrc_t from, uint32_t at)
{
    if constexpr (N == 1) to[0] = __builtin_amdgcn_raw_buffer_load_b32(from, (int)at, 0, AUX);
    else if constexpr (N == 2) { const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(from, (int)at, 0, AUX); to[0] = x[0]; to[1] = x[1]; }
    else { const u32x4_t x = __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 0, AUX); to[0] = x[0]; to[1] = x[1]; to[2] = x[2]; to[3] = x[3]; }
}

// The operand for dimension i of a lane's DL: 8 tokens' elements of it.
template <int FMT, int VW> __device__ __forceinline__ u32x4_t value_operand(const uint32_t (&v)[8][VW], int i)
{
    u32x4_t r;
#pragma unroll
    for (int p = 0; p < 4; p++) {
        if constexpr (FMT == ZC_FMT_BF16) {
            r[p] = __builtin_amdgcn_perm(v[2 * p + 1][i / 2], v[2 * p][i / 2], (i & 1) ? 0x07060302u : 0x05040100u);
        } else {
            const uint32_t w = __builtin_amdgcn_perm(v[2 * p + 1][i / 4], v[2 * p][i / 4], (i & 2) ? 0x07030602u : 0x05010400u);
            r[p] = (i & 1) ? two_to_half<FMT, true>(w) : two_to_half<FMT, false>(w);
        }
    }
    return r;
}

// The same for FP4, dimensions 2 SEL and 2 SEL + 1.  MX: every token's pair of them is converted with its scale, then the tokens are paired.  NV: the
// tokens are paired first, four bits each to a byte (`pairs`: of even dimensions, then of odd ones), converted, and multiplied with the two scales.
// my_block: where the lane's scale is in its tokens' words of them, in bits.
template <int FMT, int D, int SEL> __device__ __forceinline__ void value_operands4(const uint32_t (&v)[8], const uint32_t (&scale)[8], const uint32_t (&pairs)[4][2], uint32_t my_block, u32x4_t &even, u32x4_t &odd)
{
#pragma unroll
    for (int p = 0; p < 4; p++) {
        if constexpr (FMT == ZC_FMT_FP4_E2M1_NV) {
            const halfx2 s = __builtin_bit_cast(halfx2, two_to_half<ZC_FMT_FP8_E4M3, false>(
                kRowScales<FMT, D> == 4 ? __builtin_amdgcn_perm(scale[2 * p + 1], scale[2 * p], my_block / 8 * 0x0101u + 0x0400u) : scale[2 * p + 1] << 8 | scale[2 * p]));
            even[p] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(halfx2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(pairs[p][0], 1.0f, SEL)) * s);
            odd[p] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(halfx2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(pairs[p][1], 1.0f, SEL)) * s);
            continue;
        }
        // (the byte comes to the exponent's place; sign and mantissa beside it do not count)
        auto factor = [&](uint32_t x) { return __uint_as_float(kRowScales<FMT, D> == 4 ? __builtin_amdgcn_alignbit(x, x, my_block + 9) : x << 23); };
        const uint32_t a = two_fp4_to_values<FMT, SEL>(v[2 * p], factor(scale[2 * p])), b = two_fp4_to_values<FMT, SEL>(v[2 * p + 1], factor(scale[2 * p + 1]));
        even[p] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        odd[p] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    }
}

template <int D, int QT, uint32_t WAVES = kWaves> struct FewShared {
    float ml[WAVES][QT * 16][2];
    alignas(16) float ob[WAVES][16][D + 4];
};

// Blocks of 32 tokens that a part of `count` of them has: steps that all wavefronts take part in.
template <uint32_t WAVES> __device__ __forceinline__ int32_t blocks_per_part(const AttendDev &a, int32_t count)
{
    const int32_t even = min((count + (int32_t)a.even - 1) / (int32_t)a.even, (int32_t)a.long_part / 32), least = (count + (int32_t)a.splits - 1) / (int32_t)a.splits;
    return (max(even, least) + (int32_t)WAVES - 1) / (int32_t)WAVES * (int32_t)WAVES;
}

// Whether a call whose pages may go past the caches (plan_attend) has them do so, for one part of one (sequence, head): all sequences together have more
// tokens than a.past_caches, counting those that are read (of many sequences by the next 256), and the page in the middle of them is not also the next 64
// sequences' (which would find it in the caches).  A part of less than kLeastChoice tokens does not wait for that.
__device__ __forceinline__ bool past_caches(const AttendDev &a, uint32_t unit, uint32_t split)
{
    const uint32_t lane = threadIdx.x & 63, head = unit % a.c.heads, seq = unit / a.c.heads, n = min(a.n_seqs, 256u);
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit), read = min(length, a.reach);
    const int32_t blocks = (read + 31) / 32, per_part = blocks_per_part<kWaves>(a, blocks);
    if (min(blocks - (int32_t)split * per_part, per_part) * 32 < kLeastChoice) return false;
    auto behind = [&](uint32_t i) { return seq + i < a.n_seqs ? seq + i : seq + i - a.n_seqs; };     // the i-th sequence behind this one, i below n_seqs
    float tokens = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < 4; i++)
        if (i * 64 + lane < n) tokens += (float)clamped_length(a.c.lengths, behind(i * 64 + lane), a.reach);
    const uint32_t middle = (uint32_t)(length - (read + 1) / 2) >> a.c.page_shift;
    const uint32_t other = lane + 1 < a.n_seqs ? behind(lane + 1) : seq;
    const int32_t mine = a.c.table[(uint64_t)unit * a.c.table_pages + middle], its = a.c.table[((uint64_t)other * a.c.heads + head) * a.c.table_pages + middle];
    return !__any(other != seq && its == mine) && uniform(sum_over_wave(tokens) > (float)a.past_caches * ((float)n / (float)a.n_seqs) ? 1 : 0);
}

// PAST: pages go past the caches
constexpr int kNonTemporal = 2;                // the bit of buffer loads

template <int FMT, int D, int QT, bool LOGITS, bool PAST, uint32_t WAVES = kWaves>
__device__ __forceinline__ void attend_few(const AttendDev &a, uint32_t unit, uint32_t split, uint32_t row_block, FewShared<D, QT, WAVES> &shared)
{
    using Regs = typename FewRegs<FMT, D>::Type;
    constexpr int DL = Regs::DL, KS = D / 32;
    constexpr uint32_t kRow = kRowBytes<FMT, D>;
    constexpr int AUX = PAST ? kNonTemporal : 0;
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const uint32_t head = unit % a.c.heads, seq = unit / a.c.heads;              // a shared prefix's one "sequence" is 0

    // ---- this lane's rows, and what all of them and any of them see
    const int32_t prefix = prefix_tokens(a), offset = a.shared ? 0 : prefix;
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit);
    const Span span = rows_span(a, seq);
    const int32_t sinks = (int32_t)a.sinks - offset;
    Row rows[QT];
    const uint32_t first_row = row_block * QT * 16;
    int32_t first = 0, last = span.count - 1;            // query tokens of the sequence that the rows belong to
    if (a.row_blocks > 1) {
        first = (int32_t)(first_row / a.group);
        last = min((int32_t)((first_row + QT * 16 - 1) / a.group), last);
    }
    int32_t last_min = length - span.count + first, last_max = first <= last ? length - span.count + last : -1;
    int32_t from_min = a.window ? last_min - (int32_t)a.window + 1 : 0, from_max = a.window ? last_max - (int32_t)a.window + 1 : 0;
#pragma unroll
    for (int t = 0; t < QT; t++) rows[t] = row_of(a, span, head, first_row + t * 16 + n16, prefix, offset, length);
    if (a.shared) {
        last_min = INT32_MAX, last_max = -1, from_min = INT32_MAX, from_max = INT32_MIN;
#pragma unroll
        for (int t = 0; t < QT; t++)
            if (rows[t].token >= 0) {
                last_min = min(last_min, rows[t].sight.last);
                last_max = max(last_max, rows[t].sight.last);
                from_min = min(from_min, rows[t].sight.from);
                from_max = max(from_max, rows[t].sight.from);
            }
        last_min = min_over_wave(last_min);
        last_max = max_over_wave(last_max);
        from_min = min_over_wave(from_min);
        from_max = max_over_wave(from_max);
    }
    const Blocks blocks = seen_blocks(32, last_max, from_min, sinks);
    // this workgroup's part, in steps that all wavefronts take part in
    const int32_t per_split = blocks_per_part<WAVES>(a, blocks.count);
    const int32_t begin = min((int32_t)split * per_split, blocks.count), end = min(begin + per_split, blocks.count);
    if (begin == end && !a.direct) {                     // nothing left for this part (k_attend_join does not look at what its rows would be)
        const uint32_t r = first_row + threadIdx.x, i = r / a.group;
        if (threadIdx.x < QT * 16 && (int32_t)i < span.count) {
            const uint64_t slot = (uint64_t)(a.first_slot + split) * a.n_tokens * a.q_heads + (uint64_t)(span.first + (int32_t)i) * a.q_heads + head * a.group + r % a.group;
            a.part_ml[slot * 2] = kNegInf;
            a.part_ml[slot * 2 + 1] = 0.0f;
        }
        return;
    }

    const int32_t *table = a.c.table + (uint64_t)(unit) * a.c.table_pages;
    const uint32_t page_mask = (1u << a.c.page_shift) - 1;
    [[maybe_unused]] const uint32_t my_block = kFp4<FMT> && kRowScales<FMT, D> == 4 ? n16 / 4 * 8 : 0;
    const uint32_t k_lane = n16 * kRow + g * (kFp4<FMT> ? kRow / 4 : 16), v_lane = g * 4 * kRow + n16 * (kRow / 16);

    // page ids of the wavefront's next 32 steps: lane 2i + h has that of half h of step i (-1: absent)
    int32_t ids = -1, ids_from = begin + (int32_t)wave;
    auto fetch_ids = [&](int32_t b) {
        const int32_t mine = b + (int32_t)(lane >> 1) * (int32_t)WAVES;
        const uint32_t page = ((uint32_t)blocks.at(mine) * 32 + (lane & 1) * 16) >> a.c.page_shift;
        ids = -1;
        if (mine < end && page < a.c.table_pages) ids = table[page];
        if ((uint32_t)ids >= a.c.n_pages) ids = -1;
        ids_from = b;
    };
    int32_t b = begin + (int32_t)wave;
    if (b < end) fetch_ids(b);

    const float k_scale = a.c.k_scales ? a.c.k_scales[unit] : 1.0f;
    const float v_scale = a.c.v_scales ? a.c.v_scales[unit] : 1.0f;
    const float signed_c = a.scale * k_scale * kLog2e;
    // logits in base 2 (for signs and NaN see query_operand)
    const float c = fmaxf(fabsf(signed_c), kLeastFactor);

    u32x4_t q[QT][KS];
#pragma unroll
    for (int t = 0; t < QT; t++) {
        const uint16_t *row = a.q + (uint64_t)max(rows[t].token, 0) * a.q_token_stride + (uint64_t)rows[t].q_head * a.q_head_stride;
#pragma unroll
        for (int s = 0; s < KS; s++) {
            // the dimensions that the lane's piece of a key has
            const int dim = FMT == ZC_FMT_BF16 ? s * 32 + (int)g * 8 : kFp4<FMT> ? (int)g * (D / 4) + s * 8 : (s / 2) * 64 + (int)g * 16 + (s & 1) * 8;
            u32x4_t x = {0, 0, 0, 0};
            if (rows[t].token >= 0) x = *reinterpret_cast<const u32x4_t *>(row + dim);
            q[t][s] = query_operand(x, signed_c);
        }
    }

    float base[QT], l[QT];                               // what the rows' logits are taken relative to; sum over this lane's tokens
    f32x4 o[QT][DL];
#pragma unroll
    for (int t = 0; t < QT; t++) {
        base[t] = kNoBase;
        l[t] = 0.0f;
#pragma unroll
        for (int i = 0; i < DL; i++) o[t][i] = f32x4{0, 0, 0, 0};
    }

    // The two halves of a step: what of the pools they are (nothing where a page is absent or the step is none: such loads give 0
    // without going to memory), and which are present.
    struct Place { uint64_t at[2]; int32_t t0; uint32_t there; };          // at: rows of the pools
    auto place_of = [&](int32_t b) {
        Place x = {{0, 0}, 0, 0};
        if (b >= end) return x;
        if (b - ids_from >= 32 * (int32_t)WAVES) fetch_ids(b);
        const int32_t i = (b - ids_from) / (int32_t)WAVES * 2;
        x.t0 = blocks.at(b) * 32;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int32_t page = __builtin_amdgcn_readlane(ids, i + h);
            x.there |= page >= 0 ? 1u << h : 0u;
            x.at[h] = ((uint64_t)(uint32_t)max(page, 0) << a.c.page_shift) + (((uint32_t)x.t0 + h * 16) & page_mask);
        }
        return x;
    };
    auto load_keys = [&](const Place &x, Regs &r) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const __amdgpu_buffer_rsrc_t from = sixteen_tokens(a.c.k + x.at[h] * kRow, x.there >> h & 1 ? 16 * kRow : 0);
            if constexpr (kFp4<FMT>) {
                constexpr uint32_t kScales = kRowScales<FMT, D>;
                const __amdgpu_buffer_rsrc_t scales = sixteen_tokens(a.c.k_blocks + x.at[h] * kScales, x.there >> h & 1 ? 16 * kScales : 0);
                load_words<AUX>(r.k[h], from, k_lane);
                // a quarter of a key has two scales, one, or half of one
                if constexpr (kScales == 8) r.k_scale[h] = __builtin_amdgcn_raw_buffer_load_b16(scales, (int)(n16 * 8 + g * 2), 0, 0);
                else r.k_scale[h] = __builtin_amdgcn_raw_buffer_load_b8(scales, (int)(n16 * kScales + g * kScales / 4), 0, 0);
            } else {
#pragma unroll
                for (int u = 0; u < Regs::NK; u++) r.k[h][u] = __builtin_amdgcn_raw_buffer_load_b128(from, (int)(k_lane + u * 64), 0, AUX);
            }
        }
    };
    auto load_values = [&](const Place &x, Regs &r) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const __amdgpu_buffer_rsrc_t from = sixteen_tokens(a.c.v + x.at[h] * kRow, x.there >> h & 1 ? 16 * kRow : 0);
            if constexpr (kFp4<FMT>) {
                constexpr uint32_t kScales = kRowScales<FMT, D>;
                const __amdgpu_buffer_rsrc_t scales = sixteen_tokens(a.c.v_blocks + x.at[h] * kScales, x.there >> h & 1 ? 16 * kScales : 0);
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    if constexpr (kScales == 4) break;
                    r.v_scale[h * 4 + j] = __builtin_amdgcn_raw_buffer_load_b8(scales, (int)((g * 4 + j) * kScales + n16 * kScales / 16), 0, 0);
                }
                if constexpr (kScales == 4) {            // all of a token's four scales
                    const u32x4_t x = __builtin_amdgcn_raw_buffer_load_b128(scales, (int)(g * 16), 0, 0);
#pragma unroll
                    for (int j = 0; j < 4; j++) r.v_scale[h * 4 + j] = x[j];
                }
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    if constexpr (DL == 8) r.v[h * 4 + j] = __builtin_amdgcn_raw_buffer_load_b32(from, (int)(v_lane + j * kRow), 0, AUX);
                    else r.v[h * 4 + j] = __builtin_amdgcn_raw_buffer_load_b16(from, (int)(v_lane + j * kRow), 0, AUX);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) load_words<AUX>(r.v[h * 4 + j], from, v_lane + j * kRow);
            }
        }
    };

    // Keys of the next step are asked for when this step's products are on their way, values when this step's are used up.  (Three
    // steps ahead in as many sets of registers was slower: three copies of the loop to fetch, and a step or two is what a wavefront has.)
    Regs r;
    Place place = place_of(b);
    load_keys(place, r);
    load_values(place, r);
    for (; b < end; b += (int32_t)WAVES) {
        const int32_t t0 = place.t0;
        const uint32_t there = place.there;
        place = place_of(b + (int32_t)WAVES);
        f32x4 s[QT][2];
#pragma unroll
        for (int t = 0; t < QT; t++) s[t][0] = s[t][1] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < 2; h++) {
#pragma unroll
            for (int u = 0; u < KS; u++) {
                u32x4_t key;
                if constexpr (kFp4<FMT>) key = eight_fp4_to_bf16<FMT>(r.k[h][u], block_scale<FMT>(kRowScales<FMT, D> == 8 && u >= 2 ? r.k_scale[h] >> 8 : r.k_scale[h] & 0xFFu));
                else if constexpr (FMT == ZC_FMT_BF16) key = r.k[h][u];
                else key = eight_to_bf16<FMT>(r.k[h][u / 2][(u & 1) * 2], r.k[h][u / 2][(u & 1) * 2 + 1]);
#pragma unroll
                for (int t = 0; t < QT; t++) s[t][h] = mma16_keys(key, q[t][u], s[t][h]);
            }
        }
        load_keys(place, r);
        const bool whole = there == 3 && t0 + 31 <= last_min && (t0 >= from_max || t0 + 32 <= sinks);
        uint32_t bad = 0;                                // bit j: token j of this lane's 8 has an element that is not finite
        if (__builtin_expect(!whole, 0)) {
            // Tokens that no row sees are zeroed (what they hold is not to be multiplied, not even with 0); of those that only some
            // rows see, elements that are not finite are zeroed too and added to the rows that do see them below.
            const uint32_t halves = (there & 1 ? 0x0Fu : 0u) | (there & 2 ? 0xF0u : 0u);
            const uint32_t used = halves & seen_of_eight(Sight{last_max, from_min, sinks}, t0 + (int32_t)g * 4);
            const uint32_t by_all = seen_of_eight(Sight{last_min, from_max, sinks}, t0 + (int32_t)g * 4);
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const uint32_t keep = bit_as_mask(used, j), some = ~bit_as_mask(by_all, j);
                if constexpr (kFp4<FMT>) {               // (a scale that is not finite takes its block's elements along)
                    const uint32_t scale = r.v_scale[j] & keep, wild = wild_scale<FMT>(scale >> my_block & 0xFFu) ? some : 0u;
                    bad |= wild ? 1u << j : 0u;
                    r.v_scale[j] = scale & ~wild;
                    r.v[j] &= keep & ~wild;
                } else {
#pragma unroll
                    for (int w = 0; w < Regs::VW; w++) {
                        const uint32_t x = r.v[j][w] & keep, wild = nonfinite_mask<FMT>(x) & some;
                        bad |= wild ? 1u << j : 0u;
                        r.v[j][w] = x & ~wild;
                    }
                }
            }
        }
        u32x4_t p[QT];
#pragma unroll
        for (int t = 0; t < QT; t++) {
            if (__builtin_expect(!whole, 0)) {
                const uint32_t mask = seen_of_eight(rows[t].sight, t0 + (int32_t)g * 4) & ((there & 1 ? 0x0Fu : 0u) | (there & 2 ? 0xF0u : 0u));
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const uint32_t keep = bit_as_mask(mask, j);
                    s[t][j / 4][j & 3] = __uint_as_float((bits(s[t][j / 4][j & 3]) & keep) | (bits(kNegInf) & ~keep));
                }
            }
            if (LOGITS && rows[t].token >= 0) {
                float *to = a.logits + ((uint64_t)unit * a.logit_rows + t * 16 + n16) * a.logit_stride + (uint32_t)t0 + g * 4;
#pragma unroll
                for (int h = 0; h < 2; h++) *reinterpret_cast<f32x4 *>(to + h * 16) = s[t][h] * c;
            }
            float top = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])), fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
            top = max_over_16(max_over_32(top));
            if (__any(out_of_reach<FMT>(base[t], top, c))) {
                const float now = raised<FMT>(base[t], top, c);
                const float f = __builtin_amdgcn_exp2f(base[t] - now);
                base[t] = now;
                l[t] *= f;
#pragma unroll
                for (int i = 0; i < DL; i++) o[t][i] *= f;
            }
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; j++) e[j] = weight_of(s[t][j / 4][j & 3], c, base[t]);
            l[t] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
#pragma unroll
            for (int j = 0; j < 4; j++) p[t][j] = pack_weights<FMT>(e[2 * j], e[2 * j + 1]);
            if (__builtin_expect(__any(bad != 0), 0)) {
#pragma unroll 1
                for (uint32_t n = 0; n < 32; n++) {      // token 4 gg + (j & 3) of half j / 4
                    const uint32_t j = n & 7, gg = n >> 3;
                    if (!__any((bad >> j & 1) && g == gg)) continue;
                    const int32_t tok = t0 + (int32_t)(j / 4 * 16 + gg * 4 + (j & 3));
                    float weight = e[0];
#pragma unroll
                    for (uint32_t k = 1; k < 8; k++) weight = j == k ? e[k] : weight;
                    weight = __shfl(weight, (int)(n16 + gg * 16));
                    const bool mine = seen(rows[t].sight, tok);
                    const uint64_t stored = ((uint64_t)(uint32_t)max(table[(uint32_t)tok >> a.c.page_shift], 0) << a.c.page_shift) + ((uint32_t)tok & page_mask);
#pragma unroll
                    for (int cc = 0; cc < 4; cc++) {
#pragma unroll
                        for (int i = 0; i < DL; i += 4) {
                            const f32x4 x = wild_values<FMT, D>(a.c, stored, (g * 4 + cc) * DL + i);
#pragma unroll
                            for (int n4 = 0; n4 < 4; n4++) o[t][i + n4][cc] += mine && x[n4] != 0.0f ? weight * x[n4] : 0.0f;
                        }
                        __builtin_amdgcn_sched_barrier(0);       // a few at a time: this hardly ever runs and is to cost no registers
                    }
                }
            }
        }
        if constexpr (kFp4<FMT>) {
            uint32_t pairs[4][2];
            if constexpr (FMT == ZC_FMT_FP4_E2M1_NV) {
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t x = r.v[2 * i], y = r.v[2 * i + 1];
                    pairs[i][0] = (x & 0x0F0F0F0Fu) | (y << 4 & 0xF0F0F0F0u);
                    pairs[i][1] = (x >> 4 & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u);
                }
            }
#pragma unroll
            for (int i = 0; i < DL; i += 2) {
                u32x4_t even, odd;
                if (i == 0) value_operands4<FMT, D, 0>(r.v, r.v_scale, pairs, my_block, even, odd);
                else if (i == 2) value_operands4<FMT, D, 1>(r.v, r.v_scale, pairs, my_block, even, odd);
                else if (i == 4) value_operands4<FMT, D, 2>(r.v, r.v_scale, pairs, my_block, even, odd);
                else value_operands4<FMT, D, 3>(r.v, r.v_scale, pairs, my_block, even, odd);
#pragma unroll
                for (int t = 0; t < QT; t++) {
                    o[t][i] = mma16_values<FMT>(even, p[t], o[t][i]);
                    o[t][i + 1] = mma16_values<FMT>(odd, p[t], o[t][i + 1]);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < DL; i++) {
                const u32x4_t val = value_operand<FMT>(r.v, i);
#pragma unroll
                for (int t = 0; t < QT; t++) o[t][i] = mma16_values<FMT>(val, p[t], o[t][i]);
            }
        }
        load_values(place, r);
    }

    // ---- the wavefronts' results, 16 rows at a time
    auto &ml = shared.ml;
    auto &ob = shared.ob;
#pragma unroll
    for (int t = 0; t < QT; t++) {
        l[t] = sum_over_16(sum_over_32(l[t]));
        if (g == 0) { ml[wave][t * 16 + n16][0] = part_base(base[t], l[t]); ml[wave][t * 16 + n16][1] = l[t]; }
    }
    __syncthreads();
    constexpr uint32_t kPerRow = WAVES * 4, DP = D / kPerRow;     // threads per row, dimensions per thread
    const uint32_t row16 = threadIdx.x / kPerRow, piece = threadIdx.x % kPerRow;
#pragma unroll
    for (int t = 0; t < QT; t++) {
        const float mine = ml[wave][t * 16 + n16][0];
        float top = kNegInf;
#pragma unroll
        for (uint32_t w = 0; w < WAVES; w++) top = fmaxf(top, ml[w][t * 16 + n16][0]);
        const float f = __builtin_amdgcn_exp2f(mine - (top == kNegInf ? 0.0f : top));
#pragma unroll
        for (int cc = 0; cc < 4; cc++)
#pragma unroll
            for (int i = 0; i < DL; i += 4) {
                f32x4 x;
#pragma unroll
                for (int j = 0; j < 4; j++) x[j] = o[t][i + j][cc] * f;
                *reinterpret_cast<f32x4 *>(&ob[wave][n16][((int)g * 4 + cc) * DL + i]) = x;
            }
        __syncthreads();
        {
            const uint32_t r = first_row + t * 16 + row16, i = r / a.group;
            int32_t tok = (int32_t)i < span.count ? span.first + (int32_t)i : -1;
            if (a.shared && tok >= 0 && sequence_of(a, tok) < 0) tok = -1;
            float big = kNegInf, sum = 0.0f;
#pragma unroll
            for (uint32_t w = 0; w < WAVES; w++) big = fmaxf(big, ml[w][t * 16 + row16][0]);
#pragma unroll
            for (uint32_t w = 0; w < WAVES; w++) sum += ml[w][t * 16 + row16][1] * __builtin_amdgcn_exp2f(ml[w][t * 16 + row16][0] - (big == kNegInf ? 0.0f : big));
            float x[DP];
#pragma unroll
            for (uint32_t d = 0; d < DP; d++) x[d] = 0.0f;
#pragma unroll
            for (uint32_t w = 0; w < WAVES; w++)
#pragma unroll
                for (uint32_t d = 0; d < DP; d++) x[d] += ob[w][row16][piece * DP + d];
            if (tok >= 0) {
                const uint64_t row = (uint64_t)tok * a.q_heads + head * a.group + r % a.group;
                if (a.direct) {
                    const float inv = sum == 0.0f ? 0.0f : v_scale / sum;
                    uint16_t *to = a.out + (uint64_t)tok * a.out_token_stride + (uint64_t)(head * a.group + r % a.group) * a.out_head_stride + piece * DP;
#pragma unroll
                    for (uint32_t d = 0; d < DP; d += 2) *reinterpret_cast<uint32_t *>(to + d) = pack_bf16(x[d] * inv, x[d + 1] * inv);
                    if (a.lse && piece == 0) a.lse[row] = sum == 0.0f ? kNegInf : (big + __builtin_amdgcn_logf(sum)) * kLn2;
                } else {
                    const uint64_t slot = (uint64_t)(a.first_slot + split) * a.n_tokens * a.q_heads + row;
                    float *to = a.part_o + slot * D + piece * DP;
#pragma unroll
                    for (uint32_t d = 0; d < DP; d++) to[d] = x[d] * v_scale;
                    if (piece == 0) { a.part_ml[slot * 2] = sum != sum ? sum : big; a.part_ml[slot * 2 + 1] = sum; }
                }
            }
        }
        if (t + 1 < QT) __syncthreads();
    }
}

}  // namespace zc
