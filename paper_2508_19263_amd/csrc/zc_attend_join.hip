// What follows an attention pass over K/V pages: k_attend_join puts the parts of a split cache together, k_attend_weights adds
// up the attention weight that every cached token has been given.
#include "zc_attend_device.h"

namespace zc {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
constexpr uint32_t kFewSlots = 8;

// One workgroup per (query token, query head).  With (m_s, l_s, O_s) of the slots, M = max m_s:
//   out = sum O_s 2^(m_s - M) / sum l_s 2^(m_s - M),   lse = (M + log2 of that sum) ln 2.
// A lane first holds one slot's pair (at most 64 slots), then four dimensions of every eighth (head_dim 128) or sixteenth slot.
// Bound by latency: the parts are in the L2 or the memory-side cache (128 rows of 8 slots 4 us, launch included; 2,048 rows of
// 33 slots, 35 MB, 9 us).
//
// Workgroups behind those take 1,024 tokens of a (sequence, K/V head) each and add up their weights from the logits that
// k_attend_few has left (`logits`, where rereading these costs less than rereading the keys): four tokens to a thread, eight
// rows on their way at a time.  (4 FP8 caches of 8,192 tokens, 8 K/V heads, 4 rows each: 4.5 us with the join under a kernel trace, where the
// join alone takes 4.0; the whole call 19.0 us against 16.7 without weights.)
//
// FEW: at most kFewSlots of them.  A row is D / 4 threads then, each with four dimensions of every slot, 8 or 16 rows to a workgroup, and
// nothing is exchanged: a call with 1,680 rows of 64 and three slots took 16.9 us without it and takes 15.2, one with 43,000 and two 81
// and 38.  (With the 33 slots above, 8 of them at a time would be several rounds of loads one after the other.)
template <int D, bool FEW>
__global__ __launch_bounds__(256, 4) void k_attend_join(AttendDev a, WeightsDev wt, uint32_t slots, uint32_t join_blocks, uint32_t blocks_per_unit)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint64_t n_rows = (uint64_t)a.n_tokens * a.q_heads;
    if (blockIdx.x < join_blocks) {
        constexpr uint32_t LD = D / 4, SUBS = 256 / LD;        // lanes per slot, slots at a time
        if constexpr (FEW) {
            const uint32_t row = blockIdx.x * SUBS + tid / LD, dim = tid % LD * 4;
            if (row >= n_rows) return;
            const int32_t token = (int32_t)(row / a.q_heads);
            if (sequence_of(a, token) < 0) return;
            f32x2 ml[kFewSlots];
            f32x4 part[kFewSlots];
#pragma unroll
            for (uint32_t s = 0; s < kFewSlots; s++) {
                ml[s] = f32x2{kNegInf, 0.0f};
                if (s < slots) ml[s] = *reinterpret_cast<const f32x2 *>(a.part_ml + (s * n_rows + row) * 2);
                part[s] = f32x4{0, 0, 0, 0};
                if (s < slots) part[s] = *reinterpret_cast<const f32x4 *>(a.part_o + (s * n_rows + row) * D + dim);
            }
            float top = kNegInf, sum = 0.0f;
#pragma unroll
            for (uint32_t s = 0; s < kFewSlots; s++) top = fmaxf(top, ml[s][0]);
            f32x4 x = {0, 0, 0, 0};
#pragma unroll
            for (uint32_t s = 0; s < kFewSlots; s++) {
                const float f = ml[s][0] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(ml[s][0] - top);
                sum += ml[s][0] == kNegInf ? 0.0f : ml[s][1] * f;
                x += f == 0.0f ? f32x4{0, 0, 0, 0} : part[s] * f;
            }
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const u32x2 w = {pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
            *reinterpret_cast<u32x2 *>(a.out + (uint64_t)token * a.out_token_stride + row % a.q_heads * a.out_head_stride + dim) = w;
            if (a.lse && dim == 0) a.lse[row] = sum == 0.0f ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
            return;
        }
        __shared__ f32x4 joined[4][LD];
        const uint32_t row = blockIdx.x;
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
        const float top = max_over_wave(m);
        const float f = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m - top);
        const float sum = sum_over_wave(m == kNegInf ? 0.0f : l * f);
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
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const u32x2 w = {pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
        *reinterpret_cast<u32x2 *>(a.out + (uint64_t)token * a.out_token_stride + row % a.q_heads * a.out_head_stride + dim) = w;
        if (a.lse && tid == 0) a.lse[row] = sum == 0.0f ? kNegInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
        return;
    }

    __shared__ float lse[kLogitRows];
    const uint32_t unit = (blockIdx.x - join_blocks) / blocks_per_unit, head = unit % a.c.heads, seq = unit / a.c.heads;
    const int32_t t = (int32_t)((blockIdx.x - join_blocks) % blocks_per_unit * 1024 + tid * 4);
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit);
    const Span span = query_span(a, seq);
    const uint32_t rows = (uint32_t)span.count * a.group;      // at most kLogitRows
    // the rows' lse in base 2: 16 lanes for each row's slots
    for (uint32_t r = tid / 16; r < rows; r += 16) {
        float m = kNegInf, l = 0.0f;
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
        if ((tid & 15) == 0) lse[r] = l == 0.0f ? kNegInf : m + __builtin_amdgcn_logf(l);
    }
    __syncthreads();
    if (t >= length) return;
    const Sight any = sight(a, length - 1, 0, length), first = sight(a, length - span.count, 0, length);
    // the four tokens lie in one block of those the pass has gone over, or in none
    const bool gone_over = span.count && (t + 3 >= first.from || t < any.sinks);
    f32x4 sum = {0, 0, 0, 0};
    if (gone_over) {
        const float *from = a.logits + (uint64_t)unit * a.logit_rows * a.logit_stride + (uint32_t)t;
        for (uint32_t r0 = 0; r0 < rows; r0 += 8) {            // eight rows on their way at a time
            f32x4 x[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; k++) x[k] = *reinterpret_cast<const f32x4 *>(from + (uint64_t)min(r0 + k, rows - 1) * a.logit_stride);
#pragma unroll
            for (uint32_t k = 0; k < 8; k++) {
                const float minus = r0 + k < rows ? lse[r0 + k] : kNegInf;
#pragma unroll
                for (int j = 0; j < 4; j++) sum[j] += minus == kNegInf || x[k][j] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(x[k][j] - minus);     // (hidden: minus infinity)
            }
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

// weights_out[t] = weights_in[t] + sum over the rows that see t of exp(s - lse).  A workgroup takes 256 tokens of a (sequence, K/V
// head), 64 to a wavefront, whose keys it keeps in registers, and goes over the rows that may see them 64 at a time; these come to
// LDS once for its four wavefronts, into one of two buffers while the other is worked on.  S^T = K Q^T leaves a lane one row's
// products with 32 of the tokens, whose exponentials it adds up token by token; the 32 lanes of a token are added at the end.  Where
// there are fewer workgroups than fill the GPU, `parts` of them share the tokens, each with every so many-th 64 rows, and k_weights_sum adds
// up what they leave.  The sums have one order, whatever the launch.  Bound by the matrix instructions and the exponentials: a prompt of
// 4,099 tokens, 8 K/V heads of 128 and 4 query heads to each, takes 110 us, 625 TFLOP/s, and 5 for the sums.  (Rows straight from memory to a
// wavefront's registers, each 32 bytes of 32 rows at a time: 160 us.)
template <int FMT, int D>
__global__ __launch_bounds__(256, 2) void k_attend_weights(AttendDev a, WeightsDev wt)
{
    constexpr int ES = PageElem<FMT>::BYTES, KS = D / 16;
    constexpr uint32_t kRows = 64, kPieces = D / 8, kRowsPerPass = 256 / kPieces, kPasses = kRows / kRowsPerPass;
    __shared__ __align__(1024) uint8_t lds[2][kRows * D * 2];
    __shared__ float minus_lse[2][kRows];                      // in base 2; minus infinity: the row gives nothing
    __shared__ int32_t positions[2][kRows];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), n32 = lane & 31, g = lane >> 5;
    const uint32_t units = a.n_seqs * a.c.heads, unit = blockIdx.x % units, head = unit % a.c.heads, seq = unit / a.c.heads;
    const uint32_t part = blockIdx.x / units % wt.parts;
    const int32_t block0 = (int32_t)(blockIdx.x / units / wt.parts * 256), t0 = block0 + (int32_t)wave * 64;
    const int32_t length = clamped_length(a.c.lengths, seq, a.c.limit);
    if (block0 >= length) return;                              // the whole workgroup
    const Span span = query_span(a, seq);
    const float signed_c = a.scale * (a.c.k_scales ? a.c.k_scales[unit] : 1.0f) * kLog2e;
    const float c = fmaxf(fabsf(signed_c), kLeastFactor);      // as in the passes
    const uint32_t flip = signed_c < 0 ? 0x80008000u : 0u;     // (a factor that is not a number is in every lse already)

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
    // rows that may see one of the 256 tokens: query tokens from position block0 on, up to the window's end unless some are sinks
    const int32_t before = length - span.count, first = max(0, block0 - before);
    int32_t end = span.count;
    if (a.window && block0 >= (int32_t)a.sinks) end = min(end, block0 + 255 + (int32_t)a.window - before);
    const uint32_t n_rows = (uint32_t)max(end, 0) * a.group;
    const uint32_t first_row = (uint32_t)first * a.group / kRows * kRows + part * kRows, step = kRows * wt.parts;
    float acc[32];
#pragma unroll
    for (int i = 0; i < 32; i++) acc[i] = 0.0f;

    // This thread takes a 16-byte piece of some rows of each step, and (the first 64) what goes with one of them.  A row is query token
    // `i` of the sequence, head `h` of the group; both and the place of the row are carried from step to step.
    const uint32_t piece = tid % kPieces, row0 = tid / kPieces, step_i = step / a.group, step_h = step % a.group;
    const int64_t q_token = (int64_t)a.q_token_stride, q_head = (int64_t)a.q_head_stride, back = q_token - (int64_t)a.group * q_head;
    const uint16_t *const q0 = a.q + (int64_t)span.first * q_token + (int64_t)(head * a.group) * q_head;        // the first row of all
    uint32_t i[kPasses], h[kPasses], my_i = (first_row + tid) / a.group, my_h = (first_row + tid) % a.group;
    const uint16_t *from[kPasses];
#pragma unroll
    for (uint32_t p = 0; p < kPasses; p++) {
        const uint32_t r = first_row + p * kRowsPerPass + row0;
        i[p] = r / a.group;
        h[p] = r % a.group;
        from[p] = q0 + (int64_t)i[p] * q_token + (int64_t)h[p] * q_head;
    }
    const int64_t step_q = (int64_t)step_i * q_token + (int64_t)step_h * q_head;
    u32x4_t x[kPasses];
    float my_lse = kNegInf;
    int32_t my_position = 0;
    auto fetch = [&]() {
#pragma unroll
        for (uint32_t p = 0; p < kPasses; p++) {
            const uint16_t *row = (int32_t)i[p] < end ? from[p] : q0;          // (behind the last row: some row, which gives nothing)
            x[p] = *reinterpret_cast<const u32x4_t *>(row + piece * 8);
            i[p] += step_i;
            h[p] += step_h;
            from[p] += step_q;
            if (h[p] >= a.group) { h[p] -= a.group; i[p]++; from[p] += back; }
        }
        if (tid < kRows) {
            const bool valid = (int32_t)my_i < end;
            const float v = valid ? a.lse[(uint64_t)((uint32_t)span.first + my_i) * a.q_heads + head * a.group + my_h] : kNegInf;
            my_lse = v != kNegInf ? v * -kLog2e : kNegInf;
            my_position = before + (int32_t)my_i;
            my_i += step_i;
            my_h += step_h;
            if (my_h >= a.group) { my_h -= a.group; my_i++; }
        }
    };
    auto store = [&](uint32_t buf) {
#pragma unroll
        for (uint32_t p = 0; p < kPasses; p++) *reinterpret_cast<u32x4_t *>(lds[buf] + key_place<D>(p * kRowsPerPass + row0, piece)) = x[p] ^ flip;
        if (tid < kRows) { minus_lse[buf][tid] = my_lse; positions[buf][tid] = my_position; }
    };
    auto add_up = [&](uint32_t buf) {
#pragma unroll
        for (uint32_t half = 0; half < kRows / 32; half++) {
            const uint32_t r = half * 32 + n32;
            f32x16 s[2];
            const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < KS; u++) {
                const u32x4_t q = *reinterpret_cast<const u32x4_t *>(lds[buf] + key_place<D>(r, FMT == ZC_FMT_BF16 ? u * 2 + g : (u & ~1) * 2 + g * 2 + (u & 1)));
                s[0] = mma32_keys(key[0][u], q, u ? s[0] : zero);
                s[1] = mma32_keys(key[1][u], q, u ? s[1] : zero);
            }
            float minus = minus_lse[buf][r];
            const Sight sg = sight(a, positions[buf][r], 0, length);
            // all of these rows see all of these tokens
            const bool whole = there == 15 && !__any(!(t0 + 63 <= sg.last && (t0 >= sg.from || t0 + 64 <= sg.sinks)) || minus == kNegInf);
            if (__builtin_expect(!whole, 0)) {
                uint32_t mask = 0;
#pragma unroll
                for (int n = 0; n < 8; n++) mask |= (seen_of_four(sg, t0 + n * 8 + (int32_t)g * 4) & (there >> (n / 2) & 1 ? 15u : 0u)) << (n * 4);
                mask = minus == kNegInf ? 0u : mask;
                if (__builtin_expect(__any(minus != minus), 0)) {          // a row whose softmax is not a number gives that to what it sees, and to nothing else
#pragma unroll
                    for (int k = 0; k < 32; k++) acc[k] += minus != minus && (mask >> k & 1) ? minus : 0.0f;
                    minus = minus != minus ? kNegInf : minus;
                }
#pragma unroll
                for (int k = 0; k < 32; k++) {
                    const uint32_t keep = bit_as_mask(mask, k);
                    s[k / 16][k & 15] = __uint_as_float((bits(s[k / 16][k & 15]) & keep) | (bits(kNegInf) & ~keep));
                }
            }
#pragma unroll
            for (int k = 0; k < 32; k++) acc[k] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[k / 16][k & 15], c, minus));
        }
    };
    if (first_row < n_rows) {
        fetch();
        store(0);
        fetch();
        __syncthreads();
        uint32_t buf = 0;
        for (uint32_t r0 = first_row; r0 < n_rows; r0 += step) {
            add_up(buf);
            store(buf ^ 1);                                    // (behind the last rows: of none)
            fetch();
            __syncthreads();
            buf ^= 1;
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
    // number n is token (n / 16) * 32 + (n / 4 % 4) * 8 + g * 4 + n % 4 of the wavefront's
    const int32_t t = t0 + (int32_t)(n32 / 16 * 32 + (n32 / 4 & 3) * 8 + g * 4 + (n32 & 3));
    if (t < length) {
        const uint64_t at = (uint64_t)unit * (uint64_t)a.c.capacity + (uint64_t)t;
        if (wt.parts > 1) wt.part[((uint64_t)part * units + unit) * (uint64_t)a.c.limit + (uint64_t)t] = acc[0];
        else wt.out[at] = (wt.in ? wt.in[at] : 0.0f) + acc[0];
    }
}

// A token to a thread, 256 of a (sequence, K/V head) to a workgroup: the parts' sums, one after the other.
__global__ __launch_bounds__(256) void k_weights_sum(AttendDev a, WeightsDev wt)
{
    const uint32_t units = a.n_seqs * a.c.heads, unit = blockIdx.x % units;
    const int32_t length = clamped_length(a.c.lengths, unit / a.c.heads, a.c.limit), t = (int32_t)(blockIdx.x / units * 256 + threadIdx.x);
    if (t >= length) return;
    const uint64_t at = (uint64_t)unit * (uint64_t)a.c.capacity + (uint32_t)t;
    const uint64_t from = (uint64_t)unit * (uint64_t)a.c.limit + (uint32_t)t, apart = (uint64_t)units * (uint64_t)a.c.limit;
    float x[kMostParts];
#pragma unroll
    for (uint32_t p = 0; p < kMostParts; p++) x[p] = wt.part[min(p, wt.parts - 1) * apart + from];
    float sum = 0.0f;
#pragma unroll
    for (uint32_t p = 0; p < kMostParts; p++) sum += p < wt.parts ? x[p] : 0.0f;
    wt.out[at] = (wt.in ? wt.in[at] : 0.0f) + sum;
}

template <int FMT> void launch_weights(const AttendDev &a, const WeightsDev &w, uint32_t head_dim, uint32_t blocks, hipStream_t s)
{
    if (head_dim == 64) hipLaunchKernelGGL((k_attend_weights<FMT, 64>), dim3(blocks), dim3(256), 0, s, a, w);
    else hipLaunchKernelGGL((k_attend_weights<FMT, 128>), dim3(blocks), dim3(256), 0, s, a, w);
}

}  // namespace

int launch_attend_join(const AttendDev &a, const WeightsDev &w, uint32_t head_dim, uint32_t slots, void *stream)
{
    const uint32_t rows = (uint32_t)((uint64_t)a.n_tokens * a.q_heads), per_block = slots <= kFewSlots ? 1024 / head_dim : 1;
    const uint32_t join_blocks = slots > 1 ? (rows + per_block - 1) / per_block : 0;
    const uint32_t per_unit = a.logits ? (uint32_t)(a.c.limit + 1023) / 1024 : 1, blocks = join_blocks + (a.logits ? a.n_seqs * a.c.heads * per_unit : 0);
    const hipStream_t s = (hipStream_t)stream;
    if (slots <= kFewSlots) {
        if (head_dim == 64) hipLaunchKernelGGL((k_attend_join<64, true>), dim3(blocks), dim3(256), 0, s, a, w, slots, join_blocks, per_unit);
        else hipLaunchKernelGGL((k_attend_join<128, true>), dim3(blocks), dim3(256), 0, s, a, w, slots, join_blocks, per_unit);
    } else if (head_dim == 64) hipLaunchKernelGGL((k_attend_join<64, false>), dim3(blocks), dim3(256), 0, s, a, w, slots, join_blocks, per_unit);
    else hipLaunchKernelGGL((k_attend_join<128, false>), dim3(blocks), dim3(256), 0, s, a, w, slots, join_blocks, per_unit);
    return (int)hipGetLastError();
}

int launch_attend_weights(const AttendDev &a, const WeightsDev &w, uint32_t format, uint32_t head_dim, void *stream)
{
    const uint32_t units = a.n_seqs * a.c.heads, blocks = units * w.parts * ((uint32_t)(a.c.limit + 255) / 256);
    const hipStream_t s = (hipStream_t)stream;
    if (format == ZC_FMT_BF16) launch_weights<ZC_FMT_BF16>(a, w, head_dim, blocks, s);
    else if (format == ZC_FMT_FP8_E4M3) launch_weights<ZC_FMT_FP8_E4M3>(a, w, head_dim, blocks, s);
    else launch_weights<ZC_FMT_FP8_E5M2>(a, w, head_dim, blocks, s);
    if (w.parts > 1) hipLaunchKernelGGL(k_weights_sum, dim3(units * ((uint32_t)(a.c.limit + 255) / 256)), dim3(256), 0, s, a, w);
    return (int)hipGetLastError();
}

}  // namespace zc
