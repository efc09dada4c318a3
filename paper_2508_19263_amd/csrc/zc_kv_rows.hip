// Rows of keys and values to the pages of a K/V cache and back: k_kv_write quantises as it writes, k_kv_read gives what attention
// will see, in BF16.
//
// Both read each element once and write it once.  Measured with 8 K/V heads of 128 in random pages of 16 tokens: reading 84,051 MXFP4 tokens
// 87 us, 5.0 TB/s, nearly four fifths of it writing (a large copy reaches 6.2, a fill 6.8; through the caches 95 us); 24,000 tokens BF16 36, FP8
// 24, MX 21, NV 22 us; writing these from every sixth row of a wider tensor BF16 28, MX 25 us (with inputs through the caches 2 to 6 us more), 22,617 of them
// with a scale for each sequence and head FP8 30, NV 32.  NV is bound by instructions as much as by memory: 900 of them to a wavefront for 16 rows of K
// and V, 42 us for 31,385 tokens (44 with 1,070: a reciprocal of the scale for every row, every number brought into range).  A token of each of 32
// sequences is 2.9 us of latencies one after the other, either way.
// (Rows in the order of the caller's tensors, the heads of a token in one workgroup, instead of tokens of one head, which share a page: the
// 84,051 tokens 85 -> 99 us.)
#include "zc_attend_device.h"

namespace zc {

namespace {

// A row is D / 8 lanes, eight elements to each, so a workgroup takes 2,048 / D tokens of one head, K and V, at a time, and that P times over.
template <int D> constexpr uint32_t kLanes = D / 8;
template <int D> constexpr uint32_t kTokens = 256 / kLanes<D>;

// where a lane's row lies: its (sequence, head), its number in the pools; ours: the token is a sequence's; there: so is its page
struct Place { uint32_t unit; uint64_t row; bool ours, there; };

__device__ __forceinline__ float clamped(float x, float most) { return x != x ? x : fminf(fmaxf(x, -most), most); }
constexpr float kLargest = 0x1.fffffep127f;

// what a row's K and V are multiplied with before they are stored, where the cache has scales; zero: bit 0, 1: K, V become 0
struct Factors { float of[2]; uint32_t zero; };

__device__ __forceinline__ Factors factors_of(const RowsDev &r, const Place &p)
{
    Factors f = {{1.0f, 1.0f}, 0};
#pragma unroll
    for (int kv = 0; kv < 2; kv++) {
        const float *scales = kv ? r.c.v_scales : r.c.k_scales;
        const float divisor = scales ? scales[p.unit] : 1.0f;
        f.of[kv] = divisor == 0.0f ? 1.0f : clamped(1.0f / divisor, kLargest);
        f.zero |= divisor == 0.0f ? 1u << kv : 0u;
    }
    return f;
}

// of a token whose sequence is `seq`, `before` its tokens from this one on (none where that is less than 1)
__device__ __forceinline__ Place place_of(const RowsDev &r, uint32_t head, int32_t seq, int32_t before)
{
    Place p = {0, 0, before > 0, false};
    if (!p.ours) return p;
    p.unit = (uint32_t)seq * r.c.heads + head;
    // (a length may be any number: differences of two are taken in 64 bits)
    const int64_t position = (int64_t)max(r.c.lengths[seq], 0) - before;
    if (position < 0 || position >= r.c.capacity) return p;
    const uint32_t at = (uint32_t)position;
    const int32_t page = r.c.table[(uint64_t)p.unit * r.c.table_pages + (at >> r.c.page_shift)];
    p.there = (uint32_t)page < r.c.n_pages;
    p.row = ((uint64_t)(uint32_t)page << r.c.page_shift) + (at & ((1u << r.c.page_shift) - 1));
    return p;
}
template <int LANE> __device__ __forceinline__ uint32_t of_four(uint32_t x)       // of the LANE-th of every four lanes
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, LANE * 0x55, 0xF, 0xF, false);
}
template <int LANE> __device__ __forceinline__ Place of_four(const Place &p)
{
    const uint32_t flags = of_four<LANE>((p.ours ? 1u : 0u) | (p.there ? 2u : 0u));
    return Place{of_four<LANE>(p.unit), (uint64_t)of_four<LANE>((uint32_t)(p.row >> 32)) << 32 | of_four<LANE>((uint32_t)p.row), (flags & 1) != 0, (flags & 2) != 0};
}
template <int LANE> __device__ __forceinline__ Factors of_four(const Factors &f)
{
    return Factors{{__uint_as_float(of_four<LANE>(bits(f.of[0]))), __uint_as_float(of_four<LANE>(bits(f.of[1])))}, of_four<LANE>(f.zero)};
}

// The places (TIMES: and factors) of the lane's P tokens (1 or 4), which are kTokens apart.  A row has at least eight lanes, so of four tokens each of four lanes finds one.
// The sequence is the last one that begins at or before the token: the wavefront's tokens are counted against 64 beginnings at a time (a
// binary search waits for each of its steps: it is left to many sequences, and to four tokens to a lane where a sequence ends among them).
template <int D, int P, bool TIMES> __device__ __forceinline__ void find_places(const RowsDev &r, uint32_t head, int32_t token, Place (&p)[P], Factors (&f)[P])
{
    static_assert(P == 1 || P == 4, "");
    constexpr int kEach = 64 / (int)kLanes<D>;
    const uint32_t lane = threadIdx.x & 63;
    const int32_t n = (int32_t)r.n_tokens, mine = token + (P == 4 ? (int32_t)(lane & 3) * (int32_t)kTokens<D> : 0);
    int32_t seq = mine, before = mine < n ? 1 : 0;
    if (r.q_start) {
        const int32_t first = __builtin_amdgcn_readfirstlane(token);
        int32_t lo = -1, hi = (int32_t)r.n_seqs;               // begins at or before the token; begins behind it
        if (r.n_seqs <= 1024) {
            if constexpr (P == 1) {
                for (uint32_t c = 0; c < r.n_seqs; c += 64) {
                    const int32_t begin = c + lane < r.n_seqs ? r.q_start[c + lane] : INT32_MAX;
#pragma unroll
                    for (int j = 0; j < kEach; j++) {
                        const int32_t count = (int32_t)__popcll(__ballot(begin <= first + j));
                        lo += mine == first + j ? count : 0;
                    }
                }
                hi = lo + 1;
            } else {
                const int32_t last = first + (P - 1) * (int32_t)kTokens<D> + kEach - 1;
                hi = 0;
                for (uint32_t c = 0; c < r.n_seqs; c += 64) {
                    const int32_t begin = c + lane < r.n_seqs ? r.q_start[c + lane] : INT32_MAX;
                    lo += (int32_t)__popcll(__ballot(begin <= first));
                    hi += (int32_t)__popcll(__ballot(begin <= last));
                }
            }
        }
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) / 2;
            if (r.q_start[mid] <= mine) lo = mid; else hi = mid;
        }
        seq = lo;
        before = seq >= 0 && mine < n ? min(max(r.q_start[seq + 1], 0), n) - mine : 0;
    }
    const Place q = place_of(r, head, seq, before);
    if constexpr (P == 1) p[0] = q;
    else {
        p[0] = of_four<0>(q);
        p[1] = of_four<1>(q);
        p[2] = of_four<2>(q);
        p[3] = of_four<3>(q);
    }
    if constexpr (TIMES) {
        const Factors own = factors_of(r, q);
        if constexpr (P == 1) f[0] = own;
        else {
            f[0] = of_four<0>(own);
            f[1] = of_four<1>(own);
            f[2] = of_four<2>(own);
            f[3] = of_four<3>(own);
        }
    }
}

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// the larger of two words' halves, each
__device__ __forceinline__ uint32_t max_of_halves(uint32_t x, uint32_t y)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
}
// The largest magnitude of the eight BF16 elements of each lane of a group of 1, 2 or 4, as an integer: NaN above infinity above all numbers.
template <int GROUP> __device__ __forceinline__ uint32_t largest_of_group(const u32x4_t &w)
{
    constexpr uint32_t kMagnitudes = 0x7FFF7FFFu;
    uint32_t x = max_of_halves(max_of_halves(w[0] & kMagnitudes, w[1] & kMagnitudes), max_of_halves(w[2] & kMagnitudes, w[3] & kMagnitudes));
    if constexpr (GROUP > 1) x = max_of_halves(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));    // lanes 1 0 3 2 of every four
    if constexpr (GROUP == 4) x = max_of_halves(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));   // 2 3 0 1
    return max(x >> 16, x & 0xFFFFu);
}

constexpr uint32_t kInf16 = 0x7F80u;

__device__ __forceinline__ void floats_of_bf16(const u32x4_t &w, float (&y)[8])
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        y[2 * i] = __uint_as_float(w[i] << 16);
        y[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// y / s by one reciprocal of s (the scales of NV blocks, 2^-9 to 448): the product's remainder, which the fused operation has exactly, corrects it,
// so that a quotient of few bits, as those half way between neighbours are, comes out as it is.
__device__ __forceinline__ float quotient(float y, float s, float reciprocal)
{
    const float q = y * reciprocal;
    return __builtin_fmaf(-__builtin_fmaf(q, s, -y), reciprocal, q);           // (this way round 0 keeps its sign)
}
__device__ __forceinline__ float reciprocal_of(float s)
{
    const float x = __builtin_amdgcn_rcpf(s);
    return __builtin_fmaf(__builtin_fmaf(-x, s, 1.0f), x, x);
}

// eight FP4 elements of y / scale, rounded to the nearest, ties to even, the largest where they are beyond it (`scale`: a power of two)
__device__ __forceinline__ uint32_t eight_to_fp4(const float (&y)[8], float scale)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
}
// (an element of a vector goes to a variable first: the compiler takes a bit cast of the element itself as that of the first one)
__device__ __forceinline__ bf16x2 bf16_pair(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }
__device__ __forceinline__ uint32_t eight_to_fp4(const u32x4_t &x, float scale)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bf16_pair(x[0]), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bf16_pair(x[1]), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bf16_pair(x[2]), scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bf16_pair(x[3]), scale, 3);
}

// What eight BF16 elements times `factor` (TIMES) are stored as; scale: FP4, the block's.
template <int FMT, bool TIMES> __device__ __forceinline__ u32x4_t quantised(const u32x4_t &x, float factor, uint32_t &scale)
{
    u32x4_t w = {0, 0, 0, 0};
    if constexpr (FMT == ZC_FMT_BF16 && !TIMES) return x;
    float y[8];
    floats_of_bf16(x, y);
    if constexpr (TIMES) {
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] *= factor;
    }
    if constexpr (FMT == ZC_FMT_BF16) {
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = pack_bf16(y[2 * i], y[2 * i + 1]);
    } else if constexpr (!kFp4<FMT>) {
        constexpr float kMost = FMT == ZC_FMT_FP8_E4M3 ? 448.0f : 57344.0f;
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] = clamped(y[i], kMost);
#pragma unroll
        for (int i = 0; i < 2; i++) {
            if constexpr (FMT == ZC_FMT_FP8_E4M3) {
                w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
                w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], (int)w[i], true);
            } else {
                w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(y[4 * i], y[4 * i + 1], 0, false);
                w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(y[4 * i + 2], y[4 * i + 3], (int)w[i], true);
            }
        }
    } else {
        const uint32_t top = largest_of_group<kBlock<FMT> / 8>(x);
        // (the largest magnitude's product is the products' largest magnitude)
        float largest = __uint_as_float(top << 16);
        if constexpr (TIMES) largest = fabsf(largest * factor);
        const bool nan = top > kInf16 || largest != largest;
        if constexpr (FMT == ZC_FMT_FP4_E2M1_MX) {
            // 2^(floor(log2 of the largest) - 2); an infinity counts as the largest number
            const int32_t e = (int32_t)min(bits(largest) >> 23, 254u) - 2;
            scale = nan ? 255u : (uint32_t)max(e, 0);
            if constexpr (TIMES) w[0] = eight_to_fp4(y, block_scale<FMT>(scale));
            else w[0] = eight_to_fp4(x, block_scale<FMT>(scale));
            w[0] = nan ? 0u : w[0];
        } else {
            scale = nan ? 0x7Fu : (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(quotient(fminf(largest, 6.0f * 448.0f), 6.0f, 1.0f / 6.0f), 0.0f, 0, false) & 0xFFu;
            const float s = block_scale<FMT>(scale), reciprocal = reciprocal_of(s);
            if (__any(largest > 0x1p20f)) {                      // whose quotients might not be numbers (6 times the largest scale is less than 2^12)
#pragma unroll
                for (int i = 0; i < 8; i++) y[i] = __builtin_amdgcn_fmed3f(y[i], -0x1p20f, 0x1p20f);
            }
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = quotient(y[i], s, reciprocal);
            w[0] = nan || s == 0.0f ? 0u : eight_to_fp4(y, 1.0f);
        }
    }
    return w;
}

// eight elements to memory or from it
template <int FMT> __device__ __forceinline__ void store_eight(uint8_t *to, const u32x4_t &w)
{
    if constexpr (FMT == ZC_FMT_BF16) *reinterpret_cast<u32x4_t *>(to) = w;
    else if constexpr (!kFp4<FMT>) *reinterpret_cast<u32x2 *>(to) = u32x2{w[0], w[1]};
    else *reinterpret_cast<uint32_t *>(to) = w[0];
}
template <int FMT> __device__ __forceinline__ u32x4_t load_eight(const uint8_t *from)
{
    u32x4_t w = {0, 0, 0, 0};
    if constexpr (FMT == ZC_FMT_BF16) w = *reinterpret_cast<const u32x4_t *>(from);
    else if constexpr (!kFp4<FMT>) {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(from);
        w[0] = x[0];
        w[1] = x[1];
    } else w[0] = *reinterpret_cast<const uint32_t *>(from);
    return w;
}

// Results of large calls go past the caches (84,051 tokens 94 -> 85 us; smaller ones that would stay there lose nothing: 24,000 tokens 27 -> 21).
template <int P> __device__ __forceinline__ void store_result(uint16_t *to, const u32x4_t &w)
{
    u32x4_t *x = reinterpret_cast<u32x4_t *>(to);
    if constexpr (P > 1) __builtin_nontemporal_store(w, x);
    else *x = w;
}

// Every element is multiplied with the reciprocal of the scale of its sequence and head (at most the largest number; where the scale is 0, all become
// 0), rounded to the nearest, ties to even, the largest number where it is beyond that.  NaN stays one; in an FP4 block it makes the block's scale NaN.
template <int FMT, int D, int P, bool TIMES>
__global__ __launch_bounds__(256) void k_kv_write(RowsDev r)
{
    const uint32_t head = blockIdx.x % r.c.heads, sub = threadIdx.x % kLanes<D>;
    const int32_t token = (int32_t)(blockIdx.x / r.c.heads * (P * kTokens<D>) + threadIdx.x / kLanes<D>);
    u32x4_t x[P][2];
#pragma unroll
    for (int i = 0; i < P; i++) {
        const uint64_t t = (uint64_t)min(token + i * (int32_t)kTokens<D>, (int32_t)r.n_tokens - 1);
        x[i][0] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(r.k + t * r.k_token_stride + (uint64_t)head * r.k_head_stride + sub * 8));
        x[i][1] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(r.v + t * r.v_token_stride + (uint64_t)head * r.v_head_stride + sub * 8));
    }
    Place p[P];
    Factors f[P];
    find_places<D, P, TIMES>(r, head, token, p, f);
#pragma unroll
    for (int i = 0; i < P; i++)
#pragma unroll
        for (int kv = 0; kv < 2; kv++) {
            uint32_t scale = 0;
            u32x4_t w = quantised<FMT, TIMES>(x[i][kv], TIMES ? f[i].of[kv] : 1.0f, scale);
            if constexpr (TIMES) {
                const uint32_t keep = ~bit_as_mask(f[i].zero, kv);
#pragma unroll
                for (int j = 0; j < 4; j++) w[j] &= keep;
                scale &= keep;
            }
            if (!p[i].there) continue;
            store_eight<FMT>((kv ? r.v_pages : r.k_pages) + p[i].row * kRowBytes<FMT, D> + sub * kElemBits<FMT>, w);
            if constexpr (kFp4<FMT>) {
                constexpr uint32_t kGroup = kBlock<FMT> / 8;
                if (sub % kGroup == 0) (kv ? r.v_scale_pages : r.k_scale_pages)[p[i].row * kRowScales<FMT, D> + sub / kGroup] = (uint8_t)scale;
            }
        }
}

// Element times its block's scale times that of its sequence and head, in 32 bits, rounded to BF16; 0 where the token's page is absent.
template <int FMT, int D, int P>
__global__ __launch_bounds__(256) void k_kv_read(RowsDev r)
{
    const uint32_t head = blockIdx.x % r.c.heads, sub = threadIdx.x % kLanes<D>;
    const int32_t token = (int32_t)(blockIdx.x / r.c.heads * (P * kTokens<D>) + threadIdx.x / kLanes<D>);
    Place p[P];
    Factors none[P];
    find_places<D, P, false>(r, head, token, p, none);
    u32x4_t w[P][2];
    uint32_t block[P][2];
    float s[P][2];
#pragma unroll
    for (int i = 0; i < P; i++)
#pragma unroll
        for (int kv = 0; kv < 2; kv++) {
            w[i][kv] = u32x4_t{0, 0, 0, 0};
            block[i][kv] = 0;
            s[i][kv] = 1.0f;
            if (!p[i].there) continue;
            w[i][kv] = load_eight<FMT>((kv ? r.c.v : r.c.k) + p[i].row * kRowBytes<FMT, D> + sub * kElemBits<FMT>);
            if constexpr (kFp4<FMT>) block[i][kv] = (kv ? r.c.v_blocks : r.c.k_blocks)[p[i].row * kRowScales<FMT, D> + sub / (kBlock<FMT> / 8)];
            const float *scales = kv ? r.c.v_scales : r.c.k_scales;
            if (scales) s[i][kv] = scales[p[i].unit];
        }
#pragma unroll
    for (int i = 0; i < P; i++) {
        if (!p[i].ours) continue;
        const uint64_t t = (uint64_t)(token + i * (int32_t)kTokens<D>);
#pragma unroll
        for (int kv = 0; kv < 2; kv++) {
            u32x4_t b;
            if constexpr (FMT == ZC_FMT_BF16) b = w[i][kv];
            else if constexpr (!kFp4<FMT>) b = eight_to_bf16<FMT>(w[i][kv][0], w[i][kv][1]);
            else b = eight_fp4_to_bf16<FMT>(w[i][kv][0], block_scale<FMT>(block[i][kv]));
            if (kv ? r.c.v_scales : r.c.k_scales) {            // (numbers as stored are exact in BF16: rounded once)
                float y[8];
                floats_of_bf16(b, y);
#pragma unroll
                for (int j = 0; j < 4; j++) b[j] = pack_bf16(y[2 * j] * s[i][kv], y[2 * j + 1] * s[i][kv]);
            }
            uint16_t *to = kv ? r.v + t * r.v_token_stride + (uint64_t)head * r.v_head_stride : r.k + t * r.k_token_stride + (uint64_t)head * r.k_head_stride;
            store_result<P>(to + sub * 8, b);
        }
    }
}

// Calls whose workgroups fill the GPU (eight to a compute unit) take four times as many tokens to each, whose loads are on their way together and
// whose places are found once: 84,051 MXFP4 tokens read 141 -> 95 us, 31,385 NVFP4 ones written and read 102 -> 78.
template <int FMT, int D, bool WRITE, int P> int launch_of(const RowsDev &r, hipStream_t s)
{
    constexpr uint32_t kEach = P * kTokens<D>;
    const dim3 blocks((r.n_tokens + kEach - 1) / kEach * r.c.heads);
    if constexpr (WRITE) {
        if (r.c.k_scales || r.c.v_scales) hipLaunchKernelGGL((k_kv_write<FMT, D, P, true>), blocks, dim3(256), 0, s, r);
        else hipLaunchKernelGGL((k_kv_write<FMT, D, P, false>), blocks, dim3(256), 0, s, r);
    }
    else hipLaunchKernelGGL((k_kv_read<FMT, D, P>), blocks, dim3(256), 0, s, r);
    return (int)hipGetLastError();
}
template <int FMT, int D, bool WRITE> int launch(const RowsDev &r, hipStream_t s)
{
    const uint64_t blocks = ((uint64_t)r.n_tokens + kTokens<D> - 1) / kTokens<D> * r.c.heads;
    return blocks >= 2048 ? launch_of<FMT, D, WRITE, 4>(r, s) : launch_of<FMT, D, WRITE, 1>(r, s);
}
template <int FMT, bool WRITE> int launch(const RowsDev &r, uint32_t head_dim, hipStream_t s)
{
    return head_dim == 64 ? launch<FMT, 64, WRITE>(r, s) : launch<FMT, 128, WRITE>(r, s);
}
template <bool WRITE> int launch(const RowsDev &r, uint32_t format, uint32_t head_dim, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (format == ZC_FMT_BF16) return launch<ZC_FMT_BF16, WRITE>(r, head_dim, s);
    if (format == ZC_FMT_FP8_E4M3) return launch<ZC_FMT_FP8_E4M3, WRITE>(r, head_dim, s);
    if (format == ZC_FMT_FP8_E5M2) return launch<ZC_FMT_FP8_E5M2, WRITE>(r, head_dim, s);
    if (format == ZC_FMT_FP4_E2M1_MX) return launch<ZC_FMT_FP4_E2M1_MX, WRITE>(r, head_dim, s);
    return launch<ZC_FMT_FP4_E2M1_NV, WRITE>(r, head_dim, s);
}

}  // namespace

int launch_kv_write(const RowsDev &r, uint32_t format, uint32_t head_dim, void *stream) { return launch<true>(r, format, head_dim, stream); }
int launch_kv_read(const RowsDev &r, uint32_t format, uint32_t head_dim, void *stream) { return launch<false>(r, format, head_dim, stream); }

}  // namespace zc
