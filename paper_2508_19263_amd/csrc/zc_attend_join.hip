// What follows an attention pass over K/V pages: k_attend_join puts the parts of a split cache together, k_attend_weights adds
// up the attention weight that every cached token has been given.
#include "zc_attend_device.h"

namespace zc {

namespace {

// One workgroup per (query token, query head).  With (m_s, l_s, O_s) of the slots, M = max m_s:
//   out = sum O_s 2^(m_s - M) / sum l_s 2^(m_s - M),   lse = (M + log2 of that sum) ln 2.
// A lane first holds one slot's pair (at most 64 slots), then four dimensions of every eighth (head_dim 128) or sixteenth slot.
// Bound by latency: the parts are in the L2 or the memory-side cache.
//
// Workgroups behind those take 1,024 tokens of a (sequence, K/V head) each and add up their weights from the logits that
// k_attend_few has left (`logits`, where rereading these costs less than rereading the keys): four tokens to a thread, the
// rows one after the other.
template <int D>
__global__ __launch_bounds__(256, 4) void k_attend_join(AttendDev a, WeightsDev wt, uint32_t slots, uint32_t join_blocks, uint32_t blocks_per_unit)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint64_t n_rows = (uint64_t)a.n_tokens * a.q_heads;
    if (blockIdx.x < join_blocks) {
        constexpr uint32_t LD = D / 4, SUBS = 256 / LD;        // lanes per slot, slots at a time
        __shared__ f32x4 joined[4][LD];
        const uint64_t row = blockIdx.x;
        const int32_t token = (int32_t)(row / a.q_heads);
        if (sequence_of(a, token) < 0) return;
        float m = kNegInf, l = 0.0f;
        if (lane < slots) {
            m = a.part_ml[(lane * n_rows + row) * 2];
            l = a.part_ml[(lane * n_rows + row) * 2 + 1];
        }
        const uint32_t sub = tid / LD, dim = tid % LD * 4;
        f32x4 part[64 / SUBS];
#pragma unroll
        for (uint32_t k = 0; k < 64 / SUBS; k++) {
            const uint32_t s = k * SUBS + sub;
            part[k] = f32x4{0, 0, 0, 0};
            if (s < slots) part[k] = *reinterpret_cast<const f32x4 *>(a.part_o + (s * n_rows + row) * D + dim);
        }
        float top = m;
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        const float f = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
        float sum = m == kNegInf ? 0.0f : l * f;
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t k = 0; k < 64 / SUBS; k++) {
            const float fs = __shfl(f, (int)(k * SUBS + sub));
            x += fs == 0.0f ? f32x4{0, 0, 0, 0} : part[k] * fs;
        }
#pragma unroll
        for (uint32_t d = LD; d < 64; d *= 2)
#pragma unroll
            for (int j = 0; j < 4; j++) x[j] += __shfl_xor(x[j], (int)d);
        if (lane < LD) joined[wave][lane] = x;
        __syncthreads();
        if (tid >= LD) return;
        x = (joined[0][tid] + joined[1][tid]) + (joined[2][tid] + joined[3][tid]);
        const float inv = top == kNegInf ? 0.0f : 1.0f / sum;
        const u32x2 w = {pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
        *reinterpret_cast<u32x2 *>(a.out + (uint64_t)token * a.out_token_stride + row % a.q_heads * a.out_head_stride + dim) = w;
        if (a.lse && tid == 0) a.lse[row] = top == kNegInf ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        return;
    }

    __shared__ float lse[16];
    const uint32_t unit = (blockIdx.x - join_blocks) / blocks_per_unit, head = unit % a.c.heads, seq = unit / a.c.heads;
    const int32_t t = (int32_t)((blockIdx.x - join_blocks) % blocks_per_unit * 1024 + tid * 4);
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit);
    const Span span = query_span(a, seq);
    const uint32_t rows = (uint32_t)span.count * a.group;      // at most 16
    {
        // the rows' lse in base 2: 16 lanes for each row's slots
        const uint32_t r = tid / 16;
        float m = kNegInf, l = 0.0f;
        if (r < rows) {
            const uint64_t row = (uint64_t)(span.first + (int32_t)(r / a.group)) * a.q_heads + head * a.group + r % a.group;
            if (slots == 1) {
                m = a.lse[row] * kLog2e;
                l = 1.0f;
            } else {
                float ms[4], ls[4];
#pragma unroll
                for (uint32_t k = 0; k < 4; k++) {
                    const uint32_t s = k * 16 + (tid & 15);
                    ms[k] = s < slots ? a.part_ml[(s * n_rows + row) * 2] : kNegInf;
                    ls[k] = s < slots ? a.part_ml[(s * n_rows + row) * 2 + 1] : 0.0f;
                    m = fmaxf(m, ms[k]);
                }
                for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
#pragma unroll
                for (uint32_t k = 0; k < 4; k++) l += ms[k] == kNegInf ? 0.0f : ls[k] * __builtin_amdgcn_exp2f(ms[k] - m);
                for (int d = 1; d < 16; d *= 2) l += __shfl_xor(l, d);
            }
        }
        if ((tid & 15) == 0) lse[r] = m == kNegInf ? kNegInf : m + __builtin_amdgcn_logf(l);
        __syncthreads();
    }
    if (t >= length) return;
    const Sight any = sight(a, length - 1, 0, length), first = sight(a, length - span.count, 0, length);
    // the four tokens lie in one block of those the pass has gone over, or in none
    const bool gone_over = span.count && (t + 3 >= first.from || t < any.sinks);
    f32x4 sum = {0, 0, 0, 0};
    if (gone_over) {
        const float *from = a.logits + (uint64_t)unit * a.logit_rows * a.logit_stride + (uint32_t)t;
        for (uint32_t r = 0; r < rows; r++) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(from + (uint64_t)r * a.logit_stride);
            const float minus = lse[r];
#pragma unroll
            for (int j = 0; j < 4; j++) sum[j] += minus == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(x[j] - minus);
        }
    }
    const uint64_t at = (uint64_t)unit * (uint64_t)a.c.capacity + (uint64_t)t;
    if (t + 4 <= length) {
        const f32x4 before = wt.in ? *reinterpret_cast<const f32x4u *>(wt.in + at) : f32x4{0, 0, 0, 0};
        *reinterpret_cast<f32x4u *>(wt.out + at) = before + sum;
    } else {
        for (int j = 0; j < 4 && t + j < length; j++) wt.out[at + j] = (wt.in ? wt.in[at + j] : 0.0f) + sum[j];
    }
}

// weights_out[t] = weights_in[t] + sum over the rows that see t of exp(s - lse).  A wavefront keeps the keys of 64 tokens in
// registers and goes over the rows 32 at a time, straight from memory: S^T = K Q^T leaves a lane one row's products with 32 of
// the tokens, whose exponentials it adds up token by token; the 32 lanes of a token are added at the end.  With many rows (a prompt)
// the eight wavefronts of a workgroup share the tokens and take every eighth 32 rows, and their sums are joined in LDS; else every
// wavefront has tokens of its own.  The sums have one order, whatever the launch.  Bound by the matrix instructions and the
// exponentials with many rows, by the read of the keys with few.
template <int FMT, int D>
__global__ __launch_bounds__(512) void k_attend_weights(AttendDev a, WeightsDev wt, uint32_t by_rows)
{
    constexpr int ES = PageElem<FMT>::BYTES, KS = D / 16;
    __shared__ float sums[8][64];
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n32 = lane & 31, g = lane >> 5;
    const uint32_t units = a.n_seqs * a.c.heads, unit = blockIdx.x % units, head = unit % a.c.heads, seq = unit / a.c.heads;
    const uint32_t tile = by_rows ? blockIdx.x / units : blockIdx.x / units * (blockDim.x / 64) + wave;
    const int32_t t0 = (int32_t)(tile * 64);
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit);
    if (t0 >= length) return;                                  // by rows: the whole workgroup
    const Span span = query_span(a, seq);
    const float c = a.scale * (a.c.k_scales ? a.c.k_scales[unit] : 1.0f) * kLog2e;

    const int32_t *table = a.c.table + (uint64_t)unit * a.c.table_pages;
    const uint32_t page_log = a.c.page_shift + (D == 128 ? 7 : 6) + (ES - 1), page_mask = (1u << a.c.page_shift) - 1;
    u32x4_t key[2][KS];
    uint32_t there = 0;
#pragma unroll
    for (int h = 0; h < 4; h++) {
        const uint32_t page = ((uint32_t)t0 + h * 16) >> a.c.page_shift;
        there |= page < a.c.table_pages && (uint32_t)table[page] < a.c.n_pages ? 1u << h : 0u;
    }
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const uint32_t t = (uint32_t)t0 + h * 32 + n32, page = t >> a.c.page_shift;
        const int32_t id = page < a.c.table_pages ? table[page] : -1;
        const uint8_t *row = a.c.k + ((uint64_t)((uint32_t)id < a.c.n_pages ? id : 0) << page_log) + (t & page_mask) * (D * ES);
        // the order of the dimensions in the sums is free: FP8 keys come in pieces of 16
        if constexpr (FMT == ZC_FMT_BF16) {
#pragma unroll
            for (int u = 0; u < KS; u++) key[h][u] = *reinterpret_cast<const u32x4_t *>(row + u * 32 + g * 16);
        } else {
#pragma unroll
            for (int u = 0; u < KS; u += 2) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t *>(row + u * 16 + g * 16);
                key[h][u] = eight_to_bf16<FMT>(x[0], x[1]);
                key[h][u + 1] = eight_to_bf16<FMT>(x[2], x[3]);
            }
        }
    }
    // rows that may see one of these tokens: query tokens from position t0 on, up to the window's end unless they are sinks
    const int32_t before = length - span.count, first = max(0, t0 - before);
    int32_t end = span.count;
    if (a.window && t0 >= (int32_t)a.sinks) end = min(end, t0 + 63 + (int32_t)a.window - before);
    const uint32_t step = by_rows ? 32 * 8 : 32, first_row = (uint32_t)first * a.group + (by_rows ? wave * 32 : 0), n_rows = (uint32_t)max(end, 0) * a.group;
    float acc[32];
#pragma unroll
    for (int i = 0; i < 32; i++) acc[i] = 0.0f;

    // this lane's row of the next step: query token `i` of the sequence, head `h` of the group
    uint32_t i = (first_row + n32) / a.group, h = (first_row + n32) % a.group;
    const uint32_t step_i = step / a.group, step_h = step % a.group;
    u32x4_t q[KS];
    float lse;
    int32_t position;
    auto fetch = [&](bool valid) {
        const uint32_t tok = (uint32_t)span.first + (valid ? i : (uint32_t)first), q_head = head * a.group + h;
        const uint16_t *row = a.q + (uint64_t)tok * a.q_token_stride + (uint64_t)q_head * a.q_head_stride;
#pragma unroll
        for (int u = 0; u < KS; u++) q[u] = *reinterpret_cast<const u32x4_t *>(row + (FMT == ZC_FMT_BF16 ? u * 16 + g * 8 : (u & ~1) * 16 + g * 16 + (u & 1) * 8));
        lse = valid ? a.lse[(uint64_t)tok * a.q_heads + q_head] * kLog2e : kNegInf;
        position = before + (int32_t)i;
    };
    if (first_row < n_rows) fetch(first_row + n32 < n_rows);
    for (uint32_t r0 = first_row; r0 < n_rows; r0 += step) {
        f32x16 s[2];
#pragma unroll
        for (int k = 0; k < 16; k++) s[0][k] = s[1][k] = 0.0f;
#pragma unroll
        for (int u = 0; u < KS; u++) {
            s[0] = mma32_keys(key[0][u], q[u], s[0]);
            s[1] = mma32_keys(key[1][u], q[u], s[1]);
        }
        const Sight sg = sight(a, position, 0, length);
        const float minus = lse == kNegInf ? kNegInf : -lse;   // a row that sees nothing gives nothing
        i += step_i;
        h += step_h;
        if (h >= a.group) { h -= a.group; i++; }
        if (r0 + step < n_rows) fetch(r0 + step + n32 < n_rows);
        // all of these rows see all of these tokens
        const bool whole = there == 15 && !__any(!(t0 + 63 <= sg.last && (t0 >= sg.from || t0 + 64 <= sg.sinks)) || minus == kNegInf);
        if (whole) {
#pragma unroll
            for (int k = 0; k < 32; k++) acc[k] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[k / 16][k & 15], c, minus));
        } else {
            uint32_t mask = 0;
#pragma unroll
            for (int n = 0; n < 8; n++) mask |= (seen_of_four(sg, t0 + n * 8 + (int32_t)g * 4) & (there >> (n / 2) & 1 ? 15u : 0u)) << (n * 4);
            mask = minus == kNegInf ? 0u : mask;
#pragma unroll
            for (int k = 0; k < 32; k++) acc[k] += __uint_as_float(bits(__builtin_amdgcn_exp2f(__builtin_fmaf(s[k / 16][k & 15], c, minus))) & bit_as_mask(mask, k));
        }
    }
    // the sum over 32 lanes of each of 32 numbers: halves are exchanged until lane n has number n
#pragma unroll
    for (int width = 16; width > 0; width /= 2)
#pragma unroll
        for (int k = 0; k < width; k++) {
            const bool upper = (n32 & width) != 0;
            const float give = upper ? acc[k] : acc[k + width], keep = upper ? acc[k + width] : acc[k];
            acc[k] = keep + __shfl_xor(give, width);
        }
    // number n is token (n / 16) * 32 + (n / 4 % 4) * 8 + g * 4 + n % 4 of the tile
    const uint32_t token = n32 / 16 * 32 + (n32 / 4 & 3) * 8 + g * 4 + (n32 & 3);
    float sum = acc[0];
    if (by_rows) {
        sums[wave][token] = sum;
        __syncthreads();
        if (wave) return;
        sum = 0.0f;
        for (int w = 0; w < 8; w++) sum += sums[w][token];
    }
    const int32_t t = t0 + (int32_t)token;
    if (t < length) {
        const uint64_t at = (uint64_t)unit * (uint64_t)a.c.capacity + (uint64_t)t;
        wt.out[at] = (wt.in ? wt.in[at] : 0.0f) + sum;
    }
}

template <int FMT> void launch_weights(const AttendDev &a, const WeightsDev &w, uint32_t head_dim, uint32_t tiles, hipStream_t s)
{
    const uint32_t by_rows = (uint64_t)a.max_q_len * a.group > 64, per_group = by_rows ? 1 : 4, threads = by_rows ? 512 : 256;
    const uint32_t per_head = (tiles + per_group - 1) / per_group, blocks = a.n_seqs * a.c.heads * per_head;
    if (head_dim == 64) hipLaunchKernelGGL((k_attend_weights<FMT, 64>), dim3(blocks), dim3(threads), 0, s, a, w, by_rows);
    else hipLaunchKernelGGL((k_attend_weights<FMT, 128>), dim3(blocks), dim3(threads), 0, s, a, w, by_rows);
}

}  // namespace

int launch_attend_join(const AttendDev &a, const WeightsDev &w, uint32_t head_dim, uint32_t slots, void *stream)
{
    const uint32_t join_blocks = slots > 1 ? (uint32_t)((uint64_t)a.n_tokens * a.q_heads) : 0;
    const uint32_t per_unit = a.logits ? (uint32_t)(a.c.limit + 1023) / 1024 : 1, blocks = join_blocks + (a.logits ? a.n_seqs * a.c.heads * per_unit : 0);
    if (head_dim == 64) hipLaunchKernelGGL((k_attend_join<64>), dim3(blocks), dim3(256), 0, (hipStream_t)stream, a, w, slots, join_blocks, per_unit);
    else hipLaunchKernelGGL((k_attend_join<128>), dim3(blocks), dim3(256), 0, (hipStream_t)stream, a, w, slots, join_blocks, per_unit);
    return (int)hipGetLastError();
}

int launch_attend_weights(const AttendDev &a, const WeightsDev &w, uint32_t format, uint32_t head_dim, int32_t longest, void *stream)
{
    const uint32_t tiles = (uint32_t)(longest + 63) / 64;
    const hipStream_t s = (hipStream_t)stream;
    if (format == ZC_FMT_BF16) launch_weights<ZC_FMT_BF16>(a, w, head_dim, tiles, s);
    else if (format == ZC_FMT_FP8_E4M3) launch_weights<ZC_FMT_FP8_E4M3>(a, w, head_dim, tiles, s);
    else launch_weights<ZC_FMT_FP8_E5M2>(a, w, head_dim, tiles, s);
    return (int)hipGetLastError();
}

}  // namespace zc
