// What follows an attention pass over K/V pages: k_attend_join puts the parts of a split cache together, k_attend_weights adds
// up the attention weight that every cached token has been given.
#include "zc_attend_device.h"

namespace zc {

namespace {

// One wavefront per (query token, query head).  With (m_s, l_s, O_s) of the slots, M = max m_s:
//   out = sum O_s 2^(m_s - M) / sum l_s 2^(m_s - M),   lse = (M + log2 of that sum) ln 2.
// A lane first holds one slot's pair (at most 64 slots), then four dimensions of every second (head_dim 128) or fourth slot.
// Bound by the read of the parts, which the pass before has left in the L2 and the memory-side cache.
template <int D>
__global__ __launch_bounds__(256) void k_attend_join(AttendDev a, uint32_t slots)
{
    constexpr uint32_t LD = D / 4, SUBS = 64 / LD;
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t n_rows = (uint64_t)a.n_tokens * a.q_heads, row = (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= n_rows) return;
    const int32_t token = (int32_t)(row / a.q_heads);
    if (sequence_of(a, token) < 0) return;
    float m = kNegInf, l = 0.0f;
    if (lane < slots) {
        m = a.part_ml[(lane * n_rows + row) * 2];
        l = a.part_ml[(lane * n_rows + row) * 2 + 1];
    }
    float top = m;
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float f = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
    float sum = m == kNegInf ? 0.0f : l * f;
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    const uint32_t sub = lane / LD, dim = lane % LD * 4;
    f32x4 x = {0, 0, 0, 0};
    for (uint32_t s0 = 0; s0 < slots; s0 += SUBS * 4) {
#pragma unroll
        for (uint32_t k = 0; k < 4; k++) {
            const uint32_t s = s0 + k * SUBS + sub;
            const float fs = __shfl(f, (int)(s & 63));
            if (s < slots && fs != 0.0f) x += *reinterpret_cast<const f32x4 *>(a.part_o + (s * n_rows + row) * D + dim) * fs;
        }
    }
#pragma unroll
    for (uint32_t d = LD; d < 64; d *= 2)
#pragma unroll
        for (int j = 0; j < 4; j++) x[j] += __shfl_xor(x[j], (int)d);
    const float inv = top == kNegInf ? 0.0f : 1.0f / sum;
    if (sub == 0) {
        const u32x2 w = {pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
        *reinterpret_cast<u32x2 *>(a.out + (uint64_t)token * a.out_token_stride + row % a.q_heads * a.out_head_stride + dim) = w;
    }
    if (a.lse && lane == 0) a.lse[row] = top == kNegInf ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// weights_out[t] = weights_in[t] + sum over the rows that see t of exp(s - lse).  One wavefront per 32 tokens of a (sequence,
// K/V head), which keeps their keys in registers and goes over the rows 16 at a time: the sum has one order, whatever the launch.
template <int FMT, int D>
__global__ __launch_bounds__(256) void k_attend_weights(AttendDev a, WeightsDev wt, uint32_t blocks_per_head)
{
    constexpr int ES = PageElem<FMT>::BYTES, NK = D * ES / 64, KS = D / 32;
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const uint32_t unit = blockIdx.x / blocks_per_head, head = unit % a.c.heads, seq = unit / a.c.heads;
    const int32_t t0 = (int32_t)((blockIdx.x % blocks_per_head * 4 + wave) * 32);
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit);
    if (t0 >= length) return;
    const Span span = query_span(a, seq);
    const float signed_c = a.scale * (a.c.k_scales ? a.c.k_scales[unit] : 1.0f) * kLog2e;

    const int32_t *table = a.c.table + (uint64_t)unit * a.c.table_pages;
    const uint64_t page_bytes = (uint64_t)D * ES << a.c.page_shift;
    const uint32_t page_mask = (1u << a.c.page_shift) - 1;
    u32x4_t key[2][KS];
    bool there[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const uint32_t page = ((uint32_t)t0 + h * 16) >> a.c.page_shift;
        const int32_t id = page < a.c.table_pages ? table[page] : -1;
        there[h] = (uint32_t)id < a.c.n_pages;
        const uint8_t *p = a.c.k + (there[h] ? (uint64_t)id : 0) * page_bytes + (uint64_t)(((uint32_t)t0 + h * 16) & page_mask) * (D * ES) + n16 * (D * ES) + g * 16;
#pragma unroll
        for (int u = 0; u < NK; u++) {
            const u32x4_t x = *reinterpret_cast<const u32x4_t *>(p + u * 64);
            if constexpr (FMT == ZC_FMT_BF16) key[h][u] = x;
            else { key[h][2 * u] = eight_to_bf16<FMT>(x[0], x[1]); key[h][2 * u + 1] = eight_to_bf16<FMT>(x[2], x[3]); }
        }
    }
    // rows that may see one of these tokens: query tokens from position t0 on, up to the window's end unless they are sinks
    const int32_t before = length - span.count;
    const int32_t first = max(0, t0 - before);
    int32_t end = span.count;
    if (a.window && t0 >= (int32_t)a.sinks) end = min(end, t0 + 31 + (int32_t)a.window - before);
    float acc[2][4] = {};
    for (uint32_t r0 = (uint32_t)first * a.group; (int32_t)r0 < end * (int32_t)a.group; r0 += 16) {
        const uint32_t r = r0 + n16, i = r / a.group;
        const bool valid = (int32_t)i < end;
        const int32_t tok = span.first + (valid ? (int32_t)i : first);
        const uint32_t h = head * a.group + r % a.group;
        const uint16_t *row = a.q + (uint64_t)tok * a.q_token_stride + (uint64_t)h * a.q_head_stride;
        f32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int u = 0; u < KS; u++) {
            const int dim = FMT == ZC_FMT_BF16 ? u * 32 + (int)g * 8 : (u / 2) * 64 + (int)g * 16 + (u & 1) * 8;
            const u32x4_t x = *reinterpret_cast<const u32x4_t *>(row + dim);
#pragma unroll
            for (int hh = 0; hh < 2; hh++) s[hh] = mma16_keys(key[hh][u], x, s[hh]);
        }
        const float lse = valid ? a.lse[(uint64_t)tok * a.q_heads + h] * kLog2e : kNegInf;
        const Sight sg = sight(a, before + (int32_t)i, 0, length);
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const bool on = valid && lse != kNegInf && there[j / 4] && seen(sg, t0 + (j / 4) * 16 + (int32_t)g * 4 + (j & 3));
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j / 4][j & 3], signed_c, -lse));
            acc[j / 4][j & 3] += on ? e : 0.0f;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; j++)
#pragma unroll
        for (int d = 1; d < 16; d *= 2) acc[j / 4][j & 3] += __shfl_xor(acc[j / 4][j & 3], d);
    // lane n16 = j of each group writes token j of the group's eight
    float mine = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; j++) mine = (int)n16 == j ? acc[j / 4][j & 3] : mine;
    const int32_t t = t0 + (int32_t)(n16 / 4 * 16 + g * 4 + (n16 & 3));
    if (n16 < 8 && t < length) {
        const uint64_t at = (uint64_t)unit * (uint64_t)a.c.capacity + (uint64_t)t;
        wt.out[at] = (wt.in ? wt.in[at] : 0.0f) + mine;
    }
}

template <int FMT> void launch_weights(const AttendDev &a, const WeightsDev &w, uint32_t head_dim, uint32_t blocks, uint32_t per_head, hipStream_t s)
{
    if (head_dim == 64) hipLaunchKernelGGL((k_attend_weights<FMT, 64>), dim3(blocks), dim3(256), 0, s, a, w, per_head);
    else hipLaunchKernelGGL((k_attend_weights<FMT, 128>), dim3(blocks), dim3(256), 0, s, a, w, per_head);
}

}  // namespace

int launch_attend_join(const AttendDev &a, uint32_t head_dim, uint32_t slots, void *stream)
{
    const uint32_t blocks = (uint32_t)(((uint64_t)a.n_tokens * a.q_heads + 3) / 4);
    if (head_dim == 64) hipLaunchKernelGGL((k_attend_join<64>), dim3(blocks), dim3(256), 0, (hipStream_t)stream, a, slots);
    else hipLaunchKernelGGL((k_attend_join<128>), dim3(blocks), dim3(256), 0, (hipStream_t)stream, a, slots);
    return (int)hipGetLastError();
}

int launch_attend_weights(const AttendDev &a, const WeightsDev &w, uint32_t format, uint32_t head_dim, int32_t longest, void *stream)
{
    const uint32_t per_head = (uint32_t)(longest + 127) / 128, blocks = a.n_seqs * a.c.heads * per_head;
    if (!blocks) return 0;
    const hipStream_t s = (hipStream_t)stream;
    if (format == ZC_FMT_BF16) launch_weights<ZC_FMT_BF16>(a, w, head_dim, blocks, per_head, s);
    else if (format == ZC_FMT_FP8_E4M3) launch_weights<ZC_FMT_FP8_E4M3>(a, w, head_dim, blocks, per_head, s);
    else launch_weights<ZC_FMT_FP8_E5M2>(a, w, head_dim, blocks, per_head, s);
    return (int)hipGetLastError();
}

}  // namespace zc
