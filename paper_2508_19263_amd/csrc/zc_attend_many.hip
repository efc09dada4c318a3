// Attention over K/V pages for many query rows (prompts, batches under one prefix): k_attend_many.
//
// A workgroup of four wavefronts takes 128 (or 256) rows of one K/V head, 32 (or 64) to a wavefront, and goes over the tokens
// they see 64 at a time.  A tile of keys and values is brought to LDS once for all of them, in the type it is multiplied in (FP8
// is converted on the way: keys to BF16, values to half precision), into one of two buffers while the other is worked on:
//   S^T = K Q^T     32 tokens x 32 rows per instruction; a lane holds one row's products with half of the tile's tokens
//   O^T += V^T P^T  a lane's weights are its operand as they stand; V comes from LDS through transposing reads, four tokens
//                   of a dimension at a time, which are exactly the runs of four tokens that S^T leaves in a lane
// The bank a 16-byte piece of a key (64-byte piece of a value) lies in depends on its token too, so that neither the reads of
// 16 tokens' pieces nor the transposing ones meet in a bank.  Bound by the matrix instructions and the exponentials.
#include "zc_attend_device.h"

namespace zc {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr uint32_t kWaves = 4;
constexpr int kTile = 64;                      // tokens per step

template <int FMT> __device__ __forceinline__ f32x16 mma32_values(u32x4_t a, u32x4_t b, f32x16 c)
{
    if constexpr (FMT == ZC_FMT_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
}
template <int FMT> __device__ __forceinline__ u32x4_t eight_to_half(uint32_t lo, uint32_t hi)
{
    return u32x4_t{two_to_half<FMT, false>(lo), two_to_half<FMT, true>(lo), two_to_half<FMT, false>(hi), two_to_half<FMT, true>(hi)};
}

// Byte offsets in a tile of 64 tokens x D two-byte elements.  Keys: 16-byte piece c of a token.
template <int D> __device__ __forceinline__ uint32_t key_place(uint32_t token, uint32_t c)
{
    return D == 128 ? token * 256 + ((c ^ (token & 15)) << 4) : token * 128 + ((c ^ ((token >> 1) & 7)) << 4);
}
// Values: byte offset x inside a token's row, moved in pieces of 64 bytes.
template <int D> __device__ __forceinline__ uint32_t value_place(uint32_t token, uint32_t x)
{
    return D == 128 ? token * 256 + (x ^ ((token & 3) << 6)) : token * 128 + (x ^ ((token >> 1 & 1) << 6));
}

template <int FMT, int D, int QN>
__global__ __launch_bounds__(256, QN == 1 ? 2 : 1) void k_attend_many(AttendDev a)
{
    constexpr int ES = PageElem<FMT>::BYTES, KS = D / 16, DT = D / 32;
    constexpr uint32_t kPieces = D * ES / 16;                  // 16-byte pieces of a stored row
    constexpr uint32_t kRowsPerPass = 256 / kPieces, kPasses = kTile / kRowsPerPass;
    constexpr uint32_t kTileBytes = kTile * D * 2;
    __shared__ __align__(1024) uint8_t lds[2][2][kTileBytes];  // [buffer][keys, values]
    __shared__ uint32_t bad_tokens[3][2];                      // [tile modulo 3]: tokens with an element that is not finite
    __shared__ int32_t limits[kWaves][4];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n32 = lane & 31, g = lane >> 5;
    uint32_t id = blockIdx.x;
    const uint32_t units = (a.shared ? 1 : a.n_seqs) * a.c.heads;
    const uint32_t unit = id % units;                          // neighbours on an XCD work on the same few heads
    id /= units;
    const uint32_t split = id % a.splits, row_block = a.row_blocks - 1 - id / a.splits;    // the long rows of a prompt first
    const uint32_t head = unit % a.c.heads, seq = unit / a.c.heads;

    const int32_t prefix = prefix_tokens(a), offset = a.shared ? 0 : prefix;
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit);
    const Span span = rows_span(a, seq);
    const uint32_t first_row = row_block * (kWaves * 32 * QN);
    if ((uint64_t)first_row >= (uint64_t)span.count * a.group) return;         // the whole workgroup
    Row rows[QN];
    int32_t last_min = INT32_MAX, last_max = -1, from_min = INT32_MAX, from_max = INT32_MIN;
#pragma unroll
    for (int t = 0; t < QN; t++) {
        rows[t] = row_of(a, span, head, first_row + (wave * QN + t) * 32 + n32, prefix, offset, length);
        if (rows[t].token >= 0) {
            last_min = min(last_min, rows[t].sight.last);
            last_max = max(last_max, rows[t].sight.last);
            from_min = min(from_min, rows[t].sight.from);
            from_max = max(from_max, rows[t].sight.from);
        }
    }
    last_min = min_over_wave(last_min);
    last_max = max_over_wave(last_max);
    from_min = min_over_wave(from_min);
    from_max = max_over_wave(from_max);
    if (lane == 0) { limits[wave][0] = last_min; limits[wave][1] = last_max; limits[wave][2] = from_min; limits[wave][3] = from_max; }
    if (tid < 6) bad_tokens[tid >> 1][tid & 1] = 0;
    __syncthreads();
    // the same of the whole workgroup
    int32_t all_last_min = INT32_MAX, all_last_max = -1, all_from_min = INT32_MAX, all_from_max = INT32_MIN;
    for (uint32_t w = 0; w < kWaves; w++) {
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
    // logits in base 2; a negative factor goes to the queries' signs, and 0 is made one that takes any product to 0 but minus infinity
    const float c = fmaxf(fabsf(signed_c), 1e-30f);
    const uint32_t flip = signed_c < 0 ? 0x80008000u : 0u;
    u32x4_t q[QN][KS];
#pragma unroll
    for (int t = 0; t < QN; t++) {
        const uint16_t *row = a.q + (uint64_t)max(rows[t].token, 0) * a.q_token_stride + (uint64_t)rows[t].q_head * a.q_head_stride;
#pragma unroll
        for (int s = 0; s < KS; s++) {
            u32x4_t x = {0, 0, 0, 0};
            if (rows[t].token >= 0) x = *reinterpret_cast<const u32x4_t *>(row + s * 16 + g * 8);
            q[t][s] = x ^ flip;
        }
    }
    float m[QN], l[QN];
    f32x16 o[QN][DT];
#pragma unroll
    for (int t = 0; t < QN; t++) {
        m[t] = kNegInf;
        l[t] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[t][d][i] = 0.0f;
    }

    // ---- bringing tiles: a thread takes piece `piece` of rows row0 + pass * kRowsPerPass of keys and values
    const int32_t *table = a.c.table + (uint64_t)unit * a.c.table_pages;
    const uint32_t page_log = a.c.page_shift + (D == 128 ? 7 : 6) + (ES - 1);   // of a page's bytes
    const uint32_t page_mask = (1u << a.c.page_shift) - 1;
    const uint32_t piece = tid % kPieces, row0 = tid / kPieces;
    int32_t ids = -1, ids_from = begin;                        // lane 4i + h: page of tokens 16 h .. of tile ids_from + i (-1: absent)
    auto fetch_ids = [&](int32_t b) {
        const int32_t mine = b + (int32_t)(lane >> 2);
        const uint32_t page = ((uint32_t)blocks.at(mine) * kTile + (lane & 3) * 16) >> a.c.page_shift;
        ids = -1;
        if (mine < end && page < a.c.table_pages) ids = table[page];
        if ((uint32_t)ids >= a.c.n_pages) ids = -1;
        ids_from = b;
    };
    u32x4_t kx[kPasses], vx[kPasses];
    uint32_t fetched_there = 0;                                // of the tile in kx, vx: which of its four stretches of 16 tokens are present
    auto fetch = [&](int32_t b) {
        if (b - ids_from >= 16) fetch_ids(b);
        const int32_t at = (b - ids_from) * 4;
        const uint32_t t0 = (uint32_t)blocks.at(b) * kTile;
        fetched_there = 0;
#pragma unroll
        for (int h = 0; h < 4; h++) fetched_there |= __builtin_amdgcn_readlane(ids, at + h) >= 0 ? 1u << h : 0u;
#pragma unroll
        for (uint32_t p = 0; p < kPasses; p++) {
            const uint32_t row = p * kRowsPerPass + wave * (64 / kPieces);     // the wavefront's first: its rows lie in one stretch of 16
            const int32_t page = __builtin_amdgcn_readlane(ids, at + (int32_t)(row / 16));
            const uint64_t where = ((uint64_t)(uint32_t)max(page, 0) << page_log) + ((t0 + (row & ~15u)) & page_mask) * (D * ES);
            const uint32_t mine = ((p * kRowsPerPass + row0) & 15) * (D * ES) + piece * 16;
            kx[p] = *reinterpret_cast<const u32x4_t *>(a.c.k + where + mine);
            vx[p] = *reinterpret_cast<const u32x4_t *>(a.c.v + where + mine);
        }
    };
    // whether every row of the workgroup (of the wavefront) sees every token of a tile
    auto whole = [&](int32_t t0, uint32_t there, int32_t lmin, int32_t fmax) { return there == 15 && t0 + kTile - 1 <= lmin && (t0 >= fmax || t0 + kTile <= sinks); };
    auto store = [&](int32_t b, uint32_t buf, uint32_t mod3) {
        const int32_t t0 = blocks.at(b) * kTile;
        const bool edge = !whole(t0, fetched_there, all_last_min, all_from_max);
#pragma unroll
        for (uint32_t p = 0; p < kPasses; p++) {
            const uint32_t row = p * kRowsPerPass + row0;
            u32x4_t v = vx[p];
            if (edge) {
                // Tokens that no row sees are zeroed (what they hold is not to be multiplied, not even with 0); of those that only
                // some rows see, elements that are not finite are zeroed too and noted: they are added to the rows that do see them.
                const int32_t t = t0 + (int32_t)row;
                const bool used = (fetched_there >> (row / 16) & 1) && seen(Sight{all_last_max, all_from_min, sinks}, t);
                const bool by_all = seen(Sight{all_last_min, all_from_max, sinks}, t);
                uint32_t wild = 0;
#pragma unroll
                for (int w = 0; w < 4; w++) {
                    v[w] = used ? v[w] : 0u;
                    const uint32_t x = by_all ? 0u : nonfinite_mask<FMT>(v[w]);
                    wild |= x;
                    v[w] &= ~x;
                }
                if (wild) atomicOr(&bad_tokens[mod3][row / 32], 1u << (row & 31));
            }
            uint8_t *kt = lds[buf][0], *vt = lds[buf][1];
            if constexpr (FMT == ZC_FMT_BF16) {
                *reinterpret_cast<u32x4_t *>(kt + key_place<D>(row, piece)) = kx[p];
                *reinterpret_cast<u32x4_t *>(vt + value_place<D>(row, piece * 16)) = v;
            } else {
                *reinterpret_cast<u32x4_t *>(kt + key_place<D>(row, piece * 2)) = eight_to_bf16<FMT>(kx[p][0], kx[p][1]);
                *reinterpret_cast<u32x4_t *>(kt + key_place<D>(row, piece * 2 + 1)) = eight_to_bf16<FMT>(kx[p][2], kx[p][3]);
                *reinterpret_cast<u32x4_t *>(vt + value_place<D>(row, piece * 32)) = eight_to_half<FMT>(v[0], v[1]);
                *reinterpret_cast<u32x4_t *>(vt + value_place<D>(row, piece * 32 + 16)) = eight_to_half<FMT>(v[2], v[3]);
            }
        }
    };

    auto work = [&](int32_t b, uint32_t buf, uint32_t mod3, uint32_t there) {
        const int32_t t0 = blocks.at(b) * kTile;
        // nothing of the tile is for this wavefront's rows
        if (t0 > last_max || (t0 + kTile <= from_min && t0 >= sinks)) return;
        const uint8_t *kt = lds[buf][0], *vt = lds[buf][1];
        f32x16 s[QN][2];
#pragma unroll
        for (int t = 0; t < QN; t++)
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int i = 0; i < 16; i++) s[t][h][i] = 0.0f;
#pragma unroll
        for (int u = 0; u < KS; u++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const u32x4_t key = *reinterpret_cast<const u32x4_t *>(kt + key_place<D>(h * 32 + n32, u * 2 + g));
#pragma unroll
                for (int t = 0; t < QN; t++) s[t][h] = mma32_keys(key, q[t][u], s[t][h]);
            }
        const bool all = whole(t0, there, last_min, from_max);
        uint64_t bad = 0;
        if (!all) bad = (uint64_t)uniform(bad_tokens[mod3][0]) | (uint64_t)uniform(bad_tokens[mod3][1]) << 32;
        u32x4_t p[QN][4];
#pragma unroll
        for (int t = 0; t < QN; t++) {
            if (__builtin_expect(!all, 0)) {
                uint32_t mask = 0;                             // bit h * 16 + i: product i of half h is of a token that the row sees
#pragma unroll
                for (int n = 0; n < 8; n++) {
                    const uint32_t four = seen_of_four(rows[t].sight, t0 + n * 8 + (int32_t)g * 4) & (there >> (n / 2) & 1 ? 15u : 0u);
                    mask |= four << (n * 4);
                }
#pragma unroll
                for (int i = 0; i < 32; i++) {
                    const uint32_t keep = bit_as_mask(mask, i);
                    s[t][i / 16][i & 15] = __uint_as_float((bits(s[t][i / 16][i & 15]) & keep) | (bits(kNegInf) & ~keep));
                }
            }
            float top = s[t][0][0];
#pragma unroll
            for (int i = 1; i < 32; i++) top = fmaxf(top, s[t][i / 16][i & 15]);
            top = max_over_32(top);
            if (__any((top - m[t]) * c > kSlack)) {
                const float now = fmaxf(m[t], top);
                const float f = m[t] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f((m[t] - now) * c);
                m[t] = now;
                l[t] *= f;
#pragma unroll
                for (int d = 0; d < DT; d++) o[t][d] *= f;
            }
            const float mc = m[t] == kNegInf ? 0.0f : m[t] * c;
#pragma unroll
            for (int i = 0; i < 32; i++) {
                s[t][i / 16][i & 15] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i / 16][i & 15], c, -mc));     // (0 for the products masked above)
            }
            float sum[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 32; i++) sum[i & 3] += s[t][i / 16][i & 15];
            l[t] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            if (__builtin_expect(bad != 0, 0)) {
#pragma unroll 1
                for (uint32_t n = 0; n < 64; n++) {
                    if (!(bad >> n & 1)) continue;
                    // token n is product i of half h in the lanes of group gg
                    const uint32_t h = n >> 5, i = (n & 3) + (n >> 3 & 3) * 4, gg = n >> 2 & 1;
                    float weight = 0.0f;
#pragma unroll
                    for (uint32_t k = 0; k < 32; k++) weight = h * 16 + i == k ? s[t][k / 16][k & 15] : weight;
                    weight = __shfl(weight, (int)(n32 + gg * 32));
                    const int32_t tok = t0 + (int32_t)n;
                    const bool mine = seen(rows[t].sight, tok);
                    const uint8_t *row = a.c.v + ((uint64_t)(uint32_t)max(table[(uint32_t)tok >> a.c.page_shift], 0) << page_log) + ((uint32_t)tok & page_mask) * (D * ES);
#pragma unroll
                    for (int d = 0; d < DT; d++)
#pragma unroll
                        for (int kk = 0; kk < 16; kk += 4) {
#pragma unroll
                            for (int k = kk; k < kk + 4; k++) {
                                const float x = element<FMT>(row + (d * 32 + (k / 4) * 8 + (int)g * 4 + (k & 3)) * ES);
                                o[t][d][k] += mine && !(fabsf(x) < __builtin_inff()) ? weight * x : 0.0f;
                            }
                            __builtin_amdgcn_sched_barrier(0);   // a few at a time: this hardly ever runs and is to cost no registers
                        }
                }
            }
#pragma unroll
            for (int k = 0; k < 4; k++)
#pragma unroll
                for (int w = 0; w < 4; w++) p[t][k][w] = pack_weights<FMT>(s[t][k / 2][(k & 1) * 8 + w * 2], s[t][k / 2][(k & 1) * 8 + w * 2 + 1]);
        }
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int d = 0; d < DT; d++) {
                // lanes of a group of 16: four tokens, four 8-byte pieces of 16 dimensions
                const uint32_t tok = k * 16 + g * 4 + (lane >> 2 & 3), x = d * 64 + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + value_place<D>(tok, x)));
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(vt + value_place<D>(tok + 8, x)));
                const u32x2 lw = __builtin_bit_cast(u32x2, lo), hw = __builtin_bit_cast(u32x2, hi);
                const u32x4_t val = {lw[0], lw[1], hw[0], hw[1]};
#pragma unroll
                for (int t = 0; t < QN; t++) o[t][d] = mma32_values<FMT>(val, p[t][k], o[t][d]);
            }
    };

    if (begin < end) {
        fetch_ids(begin);
        fetch(begin);
        store(begin, 0, 0);
        uint32_t there = fetched_there;
        fetch(min(begin + 1, end - 1));
        __syncthreads();
        uint32_t mod3 = 0;
        for (int32_t b = begin; b < end; b++) {
            const uint32_t buf = (uint32_t)(b - begin) & 1, next3 = mod3 == 2 ? 0 : mod3 + 1;
            work(b, buf, mod3, there);
            if (b + 1 < end) {
                store(b + 1, buf ^ 1, next3);
                there = fetched_there;
                if (tid < 2) bad_tokens[next3 == 2 ? 0 : next3 + 1][tid] = 0;     // last read before the barrier that began this step
                fetch(min(b + 2, end - 1));                            // (the last one is asked for again: no branch, no wait)
            }
            __syncthreads();
            mod3 = next3;
        }
    }

    // ---- results: a lane has 4 consecutive dimensions at a time
#pragma unroll
    for (int t = 0; t < QN; t++) {
        if (rows[t].token < 0) continue;
        const float sum = sum_over_32(l[t]);
        const float top = m[t] == kNegInf ? kNegInf : m[t] * c;
        const uint64_t row = (uint64_t)rows[t].token * a.q_heads + rows[t].q_head;
        if (a.direct) {
            const float inv = m[t] == kNegInf ? 0.0f : v_scale / sum;
            uint16_t *to = a.out + (uint64_t)rows[t].token * a.out_token_stride + (uint64_t)rows[t].q_head * a.out_head_stride + g * 4;
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const u32x2 w = {pack_bf16(o[t][d][k * 4] * inv, o[t][d][k * 4 + 1] * inv), pack_bf16(o[t][d][k * 4 + 2] * inv, o[t][d][k * 4 + 3] * inv)};
                    *reinterpret_cast<u32x2 *>(to + d * 32 + k * 8) = w;
                }
            if (a.lse && g == 0) a.lse[row] = m[t] == kNegInf ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        } else {
            const uint64_t slot = (uint64_t)(a.first_slot + split) * a.n_tokens * a.q_heads + row;
            float *to = a.part_o + slot * D + g * 4;
#pragma unroll
            for (int d = 0; d < DT; d++)
#pragma unroll
                for (int k = 0; k < 4; k++)
                    *reinterpret_cast<f32x4 *>(to + d * 32 + k * 8) = f32x4{o[t][d][k * 4] * v_scale, o[t][d][k * 4 + 1] * v_scale, o[t][d][k * 4 + 2] * v_scale, o[t][d][k * 4 + 3] * v_scale};
            if (g == 0) { a.part_ml[slot * 2] = top; a.part_ml[slot * 2 + 1] = sum; }
        }
    }
}

template <int FMT, int D> int launch(const AttendDev &a, uint32_t tiles, uint32_t blocks, hipStream_t s)
{
    if (tiles == 1) hipLaunchKernelGGL((k_attend_many<FMT, D, 1>), dim3(blocks), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_attend_many<FMT, D, 2>), dim3(blocks), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}
template <int FMT> int launch(const AttendDev &a, uint32_t head_dim, uint32_t tiles, uint32_t blocks, hipStream_t s)
{
    return head_dim == 64 ? launch<FMT, 64>(a, tiles, blocks, s) : launch<FMT, 128>(a, tiles, blocks, s);
}

}  // namespace

int launch_attend_many(const AttendDev &a, uint32_t format, uint32_t head_dim, uint32_t tiles, void *stream)
{
    const uint32_t blocks = (a.shared ? 1 : a.n_seqs) * a.c.heads * a.row_blocks * a.splits;
    const hipStream_t s = (hipStream_t)stream;
    if (format == ZC_FMT_BF16) return launch<ZC_FMT_BF16>(a, head_dim, tiles, blocks, s);
    if (format == ZC_FMT_FP8_E4M3) return launch<ZC_FMT_FP8_E4M3>(a, head_dim, tiles, blocks, s);
    return launch<ZC_FMT_FP8_E5M2>(a, head_dim, tiles, blocks, s);
}

}  // namespace zc
