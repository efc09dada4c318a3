// Device-side helpers of the attention kernels over K/V pages: types of the matrix instructions' operands, conversion of
// page elements, positions and visibility.  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>

#include "zc_attend.h"

namespace zc {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef f32x4 f32x4u __attribute__((aligned(4)));      // where only the elements are aligned
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_inff();
// A factor of the logits of 0 would take minus infinity, which stands for what is hidden, to NaN: the smallest normal number in its place
// takes any product to less than 4, and those below 2^100 to nothing.
constexpr float kLeastFactor = 0x1p-126f;
// A row's running maximum is replaced, and what has been added up scaled, only where a weight would be more than 2^kSlack times its: the
// 32-bit sums and the operands' types (half precision to 2^16) hold what is below that with the same relative error.
constexpr float kSlack = 8.0f;
template <int FMT> constexpr bool kFp4 = FMT == ZC_FMT_FP4_E2M1_MX || FMT == ZC_FMT_FP4_E2M1_NV;
// Values are multiplied in BF16 where their range goes to no other two-byte type (BF16; MXFP4, whose scales are any power of two).
template <int FMT> constexpr bool kValuesBf16 = FMT == ZC_FMT_BF16 || FMT == ZC_FMT_FP4_E2M1_MX;
// Weights in half precision (FP8 and NVFP4 values) are all 2^kLift of what they are, and the sum that they are divided by is too.  Half
// precision ends at 2^-24, but the sum counts what is below: many light tokens beside a heavy one would lose their share.  With both
// powers weights reach 2^15 of half precision's 2^16, and end at 2^-31 of a row's heaviest.
template <int FMT> constexpr float kLift = kValuesBf16<FMT> ? 0.0f : 7.0f;

template <int FMT> constexpr int kElemBits = FMT == ZC_FMT_BF16 ? 16 : kFp4<FMT> ? 4 : 8;
template <int FMT> constexpr int kBlock = FMT == ZC_FMT_FP4_E2M1_MX ? 32 : 16;             // FP4 elements that share a scale
template <int FMT, int D> constexpr uint32_t kRowBytes = D * kElemBits<FMT> / 8;           // of a token's keys or values
template <int FMT, int D> constexpr uint32_t kRowScales = D / kBlock<FMT>;                 // FP4: bytes of a token's block scales

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint32_t bits(float x) { return __float_as_uint(x); }

// the value of the lane 32 (16) further on, combined: every lane gets f(x of it, x of that lane)
__device__ __forceinline__ float max_over_32(float x)
{
    const u32x2 r = __builtin_amdgcn_permlane32_swap(bits(x), bits(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_over_16(float x)
{
    const u32x2 r = __builtin_amdgcn_permlane16_swap(bits(x), bits(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_over_32(float x)
{
    const u32x2 r = __builtin_amdgcn_permlane32_swap(bits(x), bits(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float sum_over_16(float x)
{
    const u32x2 r = __builtin_amdgcn_permlane16_swap(bits(x), bits(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// f over all lanes of a wavefront: within rows of 16 by rotation, then over the rows
template <int N> __device__ __forceinline__ uint32_t rotated(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xF, 0xF, false); }
template <typename F> __device__ __forceinline__ uint32_t over_wave(uint32_t x, F f)
{
    x = f(x, rotated<8>(x));
    x = f(x, rotated<4>(x));
    x = f(x, rotated<2>(x));
    x = f(x, rotated<1>(x));
    u32x2 r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return f(r[0], r[1]);
}
__device__ __forceinline__ int32_t min_over_wave(int32_t x) { return uniform((int32_t)over_wave((uint32_t)x, [](uint32_t p, uint32_t q) { return (uint32_t)min((int32_t)p, (int32_t)q); })); }
__device__ __forceinline__ int32_t max_over_wave(int32_t x) { return uniform((int32_t)over_wave((uint32_t)x, [](uint32_t p, uint32_t q) { return (uint32_t)max((int32_t)p, (int32_t)q); })); }
__device__ __forceinline__ float max_over_wave(float x) { return __uint_as_float(over_wave(bits(x), [](uint32_t p, uint32_t q) { return bits(fmaxf(__uint_as_float(p), __uint_as_float(q))); })); }
__device__ __forceinline__ float sum_over_wave(float x) { return __uint_as_float(over_wave(bits(x), [](uint32_t p, uint32_t q) { return bits(__uint_as_float(p) + __uint_as_float(q)); })); }

// FP8 elements are exact in BF16 and in half precision, so keys go to the type of the queries, and values to the type with
// more mantissa: the weights they are multiplied with (at most 2^(kSlack + kLift)) are rounded to that type too.
// two bytes (the low or the high ones of a word)
template <int FMT, bool HIGH> __device__ __forceinline__ uint32_t two_to_bf16(uint32_t w)
{
    bf16x2 r;
    if constexpr (FMT == ZC_FMT_FP8_E4M3) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH);
    else r = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, HIGH);
    return __builtin_bit_cast(uint32_t, r);
}
template <int FMT, bool HIGH> __device__ __forceinline__ uint32_t two_to_half(uint32_t w)
{
    halfx2 r;
    if constexpr (FMT == ZC_FMT_FP8_E4M3) r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH);
    else r = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w, 1.0f, HIGH);
    return __builtin_bit_cast(uint32_t, r);
}
// eight FP8 elements to BF16
template <int FMT> __device__ __forceinline__ u32x4_t eight_to_bf16(uint32_t lo, uint32_t hi)
{
    return u32x4_t{two_to_bf16<FMT, false>(lo), two_to_bf16<FMT, true>(lo), two_to_bf16<FMT, false>(hi), two_to_bf16<FMT, true>(hi)};
}
// Two weights to the type the values of the format are multiplied in.  BF16 has 8 bits, and values of its range go to no other two-byte
// type: results are off by 0.0019 - 0.0022 of their norm where 32-bit weights leave the 0.0016 - 0.0017 of rounding the result (FP8 values,
// with half precision: the same 0.0017).  What is left of the weights could be multiplied too, for as many matrix instructions again.
template <int FMT> __device__ __forceinline__ uint32_t pack_weights(float a, float b)
{
    if constexpr (kValuesBf16<FMT>) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    else return __builtin_bit_cast(uint32_t, halfx2{(_Float16)a, (_Float16)b});
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }

__device__ __forceinline__ f32x4 mma16_keys(u32x4_t a, u32x4_t b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32_keys(u32x4_t a, u32x4_t b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <int FMT> __device__ __forceinline__ f32x4 mma16_values(u32x4_t a, u32x4_t b, f32x4 c)
{
    if constexpr (kValuesBf16<FMT>) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), c, 0, 0, 0);
}

// FP4 elements, two to a byte, the first in the low bits: numbers of 2 bits, times their block's scale.  MX: 2^(byte - 127), 255: NaN; the
// conversions take it as the exponent of a float (0 in its place is 2^-127, and sign and mantissa do not count).  NV: an E4M3 number.
template <int FMT> __device__ __forceinline__ float block_scale(uint32_t byte)
{
    if constexpr (FMT == ZC_FMT_FP4_E2M1_MX) return __uint_as_float(byte << 23);
    else return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
}
// whether elements of the block may be other than finite (MX: 6 times 2^126 is not)
template <int FMT> __device__ __forceinline__ bool wild_scale(uint32_t byte)
{
    if constexpr (FMT == ZC_FMT_FP4_E2M1_MX) return byte >= 253;
    else return (byte & 0x7F) == 0x7F;
}
// Elements 2 SEL and 2 SEL + 1 of a word.  To BF16 (exact: NV elements times their scale have 6 bits) and to the type that values are
// multiplied in (NV: half precision, which holds 2^-10 to 6 times 448 exactly).
template <int FMT, int SEL> __device__ __forceinline__ uint32_t two_fp4_to_bf16(uint32_t w, float scale)
{
    if constexpr (FMT == ZC_FMT_FP4_E2M1_MX) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
    else {
        const f32x2 x = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, SEL));
        return __builtin_amdgcn_perm(bits(x[1] * scale), bits(x[0] * scale), 0x07060302u);     // (nothing is cut off)
    }
}
template <int FMT, int SEL> __device__ __forceinline__ uint32_t two_fp4_to_values(uint32_t w, float scale)
{
    if constexpr (FMT == ZC_FMT_FP4_E2M1_MX) return two_fp4_to_bf16<FMT, SEL>(w, scale);
    else {
        const halfx2 x = __builtin_bit_cast(halfx2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, SEL));
        return __builtin_bit_cast(uint32_t, x * halfx2{(_Float16)scale, (_Float16)scale});
    }
}
template <int FMT> __device__ __forceinline__ u32x4_t eight_fp4_to_bf16(uint32_t w, float scale)
{
    return u32x4_t{two_fp4_to_bf16<FMT, 0>(w, scale), two_fp4_to_bf16<FMT, 1>(w, scale), two_fp4_to_bf16<FMT, 2>(w, scale), two_fp4_to_bf16<FMT, 3>(w, scale)};
}
template <int FMT> __device__ __forceinline__ u32x4_t eight_fp4_to_values(uint32_t w, float scale)
{
    return u32x4_t{two_fp4_to_values<FMT, 0>(w, scale), two_fp4_to_values<FMT, 1>(w, scale), two_fp4_to_values<FMT, 2>(w, scale), two_fp4_to_values<FMT, 3>(w, scale)};
}
// ones over those of a word's elements that are infinities or NaN
template <int FMT> __device__ __forceinline__ uint32_t nonfinite_mask(uint32_t w)
{
    static_assert(!kFp4<FMT>, "FP4 has none: see wild_scale");
    if constexpr (FMT == ZC_FMT_BF16) {
        const uint32_t t = ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;      // exponent of ones: carries into the sign's place
        return (t >> 15) * 0xFFFFu;
    } else {
        // 0x7F is E4M3's only NaN (sign aside); E5M2 has an exponent of ones
        const uint32_t t = (FMT == ZC_FMT_FP8_E4M3 ? (w & 0x7F7F7F7Fu) + 0x01010101u : (w & 0x7C7C7C7Cu) + 0x04040404u) & 0x80808080u;
        return (t >> 7) * 0xFFu;
    }
}
// Four consecutive elements of a row of values (the first a multiple of four) as floats, 0 where they are finite: what those rows that see the
// token add by themselves.  FP4: 0 only where the block's scale is not wild (its finite elements have been left out with the others).
template <int FMT, int D> __device__ __forceinline__ f32x4 wild_values(const PagesDev &c, uint64_t row, uint32_t dim)
{
    f32x4 x;
    if constexpr (kFp4<FMT>) {
        const uint32_t byte = c.v_blocks[row * kRowScales<FMT, D> + dim / kBlock<FMT>];
        const uint32_t codes = *reinterpret_cast<const uint16_t *>(c.v + row * kRowBytes<FMT, D> + dim / 2);
        const float scale = block_scale<FMT>(byte), factor = FMT == ZC_FMT_FP4_E2M1_MX ? scale : 1.0f;
        const f32x2 lo = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, factor, 0)), hi = __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, factor, 1));
        x = f32x4{lo[0], lo[1], hi[0], hi[1]};
        if constexpr (FMT == ZC_FMT_FP4_E2M1_NV) x *= scale;
        const uint32_t keep = wild_scale<FMT>(byte) ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < 4; i++) x[i] = __uint_as_float(bits(x[i]) & keep);
    } else {
        const uint8_t *p = c.v + row * kRowBytes<FMT, D> + dim * (kElemBits<FMT> / 8);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (FMT == ZC_FMT_BF16) x[i] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << 16);
            else x[i] = __uint_as_float(two_to_bf16<FMT, false>(p[i]) << 16);
            x[i] = fabsf(x[i]) < __builtin_inff() ? 0.0f : x[i];
        }
    }
    return x;
}

// 16 tokens of a page (bytes 0: none, what is asked for is 0)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t sixteen_tokens(const uint8_t *p, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(p), 0, bytes, 0x00020000);
}

// Byte offset in LDS of 16-byte piece c of row n, rows of D two-byte elements: 16 rows' pieces of one number lie in as many banks.
template <int D> __device__ __forceinline__ uint32_t key_place(uint32_t n, uint32_t c)
{
    return D == 128 ? n * 256 + ((c ^ (n & 15)) << 4) : n * 128 + ((c ^ ((n >> 1) & 7)) << 4);
}

// What a row's logits in base 2 are taken relative to, its base, is kLift below its running maximum: its weights are 2 to the power of the
// difference.  That is always taken of the base as it has been rounded, and a weight's exponent judged as it will be: of logits beyond 2^24,
// where numbers lie 2 and more apart, weights are off by powers of 2, but none leaves its type's range for that.
constexpr float kNoBase = -3e38f;              // nothing seen yet; minus infinity less it is minus infinity
template <int FMT> __device__ __forceinline__ bool out_of_reach(float base, float top, float c) { return __builtin_fmaf(top, c, -base) > kSlack + kLift<FMT>; }
// the base after a product `top`
template <int FMT> __device__ __forceinline__ float raised(float base, float top, float c) { return fmaxf(base, __builtin_fmaf(top, c, -kLift<FMT>)); }
__device__ __forceinline__ float weight_of(float product, float c, float base) { return __builtin_amdgcn_exp2f(__builtin_fmaf(product, c, -base)); }
// A part's base: minus infinity where it has seen nothing (its sum is 0), not a number where its sum is not one, though all
// its products were not numbers either and have left the base where it was.
__device__ __forceinline__ float part_base(float base, float sum) { return sum != sum ? sum : base == kNoBase ? kNegInf : base; }

// Eight elements of a query as they are multiplied: a negative factor of the logits goes to their signs, and one that is not a number takes
// their place, so that what a row sees is not a number and what is hidden from it (minus infinity, put there after the product) stays that.
__device__ __forceinline__ u32x4_t query_operand(u32x4_t x, float factor)
{
    const uint32_t flip = factor < 0 ? 0x80008000u : 0u;
    return factor != factor ? u32x4_t{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u} : x ^ flip;
}

// ---- sequences, rows, positions ----------------------------------------------------------------
struct Span { int32_t first, count; };         // a sequence's query tokens

__device__ __forceinline__ Span query_span(const AttendDev &a, uint32_t seq)
{
    if (!a.q_start) return Span{(int32_t)seq, 1};
    const int32_t n = (int32_t)a.n_tokens;
    const int32_t first = min(max(a.q_start[seq], 0), n), end = min(max(a.q_start[seq + 1], 0), n);
    return Span{first, min(max(end - first, 0), (int32_t)a.max_q_len)};
}
__device__ __forceinline__ int32_t clamped_length(const int32_t *lengths, uint32_t seq, int32_t limit) { return min(max(lengths[seq], 0), limit); }
__device__ __forceinline__ int32_t prefix_tokens(const AttendDev &a) { return a.prefix_length ? clamped_length(a.prefix_length, 0, a.prefix_limit) : 0; }

// the sequence whose query tokens include `token`, or -1
__device__ __forceinline__ int32_t sequence_of(const AttendDev &a, int32_t token)
{
    if (!a.q_start) return token;
    int32_t lo = 0, hi = (int32_t)a.n_seqs;    // the last sequence that starts at or before the token
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) / 2;
        if (a.q_start[mid] <= token) lo = mid; else hi = mid;
    }
    const Span s = query_span(a, (uint32_t)lo);
    return token >= s.first && token < s.first + s.count ? lo : -1;
}

// What a query at position p sees of a cache whose token 0 is at position `offset`, as token numbers of that cache: those up
// to `last`, of them those from `from` on and those before `sinks`.
struct Sight { int32_t last, from, sinks; };

__device__ __forceinline__ Sight sight(const AttendDev &a, int32_t position, int32_t offset, int32_t length)
{
    Sight s;
    s.last = min(position - offset, length - 1);
    s.from = a.window ? position - offset - (int32_t)a.window + 1 : 0;
    s.sinks = (int32_t)a.sinks - offset;
    return s;
}
__device__ __forceinline__ bool seen(const Sight &s, int32_t t) { return t <= s.last && (t >= s.from || t < s.sinks); }
// the low n bits, n taken into 0 .. 4
__device__ __forceinline__ uint32_t low_of_four(int32_t n) { return (1u << min(max(n, 0), 4)) - 1; }
__device__ __forceinline__ uint32_t seen_of_four(const Sight &s, int32_t t) { return low_of_four(s.last - t + 1) & (~low_of_four(s.from - t) | low_of_four(s.sinks - t)); }
// bit j: token t + j, or t + 16 + j - 4, is seen
__device__ __forceinline__ uint32_t seen_of_eight(const Sight &s, int32_t t) { return seen_of_four(s, t) | seen_of_four(s, t + 16) << 4; }
__device__ __forceinline__ uint32_t bit_as_mask(uint32_t x, int j) { return (uint32_t)__builtin_amdgcn_sbfe((int)x, j, 1); }

// A row of a (sequence, K/V head), or of a head of the shared prefix: query token r / group, query head r % group of the K/V head's.
// `span`: the query tokens the rows belong to.  token -1: there is no such row.
struct Row { int32_t token; uint32_t q_head; Sight sight; };

__device__ __forceinline__ Row row_of(const AttendDev &a, const Span &span, uint32_t head, uint32_t r, int32_t prefix, int32_t offset, int32_t length)
{
    Row x;
    const uint32_t i = r / a.group;
    x.q_head = head * a.group + r % a.group;
    x.token = (int32_t)i < span.count ? span.first + (int32_t)i : -1;
    int32_t position = 0;
    if (x.token >= 0) {
        if (a.shared) {
            const int32_t s = sequence_of(a, x.token);
            if (s < 0) x.token = -1;
            else {
                const Span own = query_span(a, (uint32_t)s);
                position = prefix + clamped_length(a.own_lengths, (uint32_t)s, a.own_limit) - own.count + (x.token - own.first);
            }
        } else position = prefix + length - span.count + (int32_t)i;
    }
    x.sight = sight(a, position, offset, length);
    return x;
}
__device__ __forceinline__ Span rows_span(const AttendDev &a, uint32_t seq) { return a.shared ? Span{0, (int32_t)a.n_tokens} : query_span(a, seq); }

// The blocks of `size` tokens that some of several rows see: those with sinks, then those from the first row's window on.
struct Blocks {
    int32_t sinks, skipped, count;             // blocks b < sinks are block b of the cache, later ones block b + skipped
    __device__ __forceinline__ int32_t at(int32_t b) const { return b < sinks ? b : b + skipped; }
};
__device__ __forceinline__ Blocks seen_blocks(int32_t size, int32_t last_max, int32_t from_min, int32_t sinks)
{
    Blocks x;
    const int32_t end = last_max < 0 ? 0 : last_max / size + 1, lo = max(from_min, 0) / size;
    x.sinks = lo > 0 ? min(min((max(sinks, 0) + size - 1) / size, lo), end) : 0;
    x.skipped = max(lo, x.sinks) - x.sinks;
    x.count = x.sinks + max(0, end - max(lo, x.sinks));
    return x;
}

}  // namespace zc
