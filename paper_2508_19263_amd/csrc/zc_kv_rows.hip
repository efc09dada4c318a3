// Rows of keys and values to the pages of a K/V cache and back: k_kv_write quantises as it writes, k_kv_read gives what attention
// will see, in BF16.
#include "zc_attend_device.h"

namespace zc {

namespace {

// A row is D / 8 lanes, eight elements to each, so a workgroup takes 2,048 / D tokens of one head, K and V.
template <int D> constexpr uint32_t kLanes = D / 8;
template <int D> constexpr uint32_t kTokens = 256 / kLanes<D>;

// where the lane's row lies: its (sequence, head), its number in the pools; ours: the token is a sequence's; there: so is its page
struct Place { uint32_t unit; uint64_t row; bool ours, there; };

template <int D> __device__ __forceinline__ Place place_of(const RowsDev &r, uint32_t head, int32_t token)
{
    const int32_t n = (int32_t)r.n_tokens;
    Place p = {0, 0, false, false};
    int32_t seq = token, before = 1;                           // tokens of the sequence from this one on
    if (r.q_start) {
        // the last sequence that begins at or before the token: the wavefront's tokens are counted against 64 beginnings at a time (a
        // binary search would wait for each of its steps)
        constexpr int kEach = 64 / (int)kLanes<D>;
        const uint32_t lane = threadIdx.x & 63;
        const int32_t first = __builtin_amdgcn_readfirstlane(token);
        seq = -1;
        if (r.n_seqs <= 1024) {
            for (uint32_t c = 0; c < r.n_seqs; c += 64) {
                const int32_t begin = c + lane < r.n_seqs ? r.q_start[c + lane] : INT32_MAX;
#pragma unroll
                for (int j = 0; j < kEach; j++) {
                    const int32_t count = (int32_t)__popcll(__ballot(begin <= first + j));
                    seq += token == first + j ? count : 0;
                }
            }
        } else {
            int32_t lo = -1, hi = (int32_t)r.n_seqs;
            while (hi - lo > 1) {
                const int32_t mid = (lo + hi) / 2;
                if (r.q_start[mid] <= token) lo = mid; else hi = mid;
            }
            seq = lo;
        }
        if (seq >= 0) before = min(max(r.q_start[seq + 1], 0), n) - token;
    }
    p.ours = token < n && seq >= 0 && before > 0;
    if (!p.ours) return p;
    // (a length may be any number: differences of two are taken in 64 bits)
    const int64_t position = (int64_t)max(r.c.lengths[seq], 0) - before;
    p.unit = (uint32_t)seq * r.c.heads + head;
    if (position < 0 || position >= r.c.capacity) return p;
    const uint32_t at = (uint32_t)position;
    const int32_t page = r.c.table[(uint64_t)p.unit * r.c.table_pages + (at >> r.c.page_shift)];
    p.there = (uint32_t)page < r.c.n_pages;
    p.row = ((uint64_t)(uint32_t)page << r.c.page_shift) + (at & ((1u << r.c.page_shift) - 1));
    return p;
}

// the largest of the lanes of a group of 2 or 4
template <int GROUP> __device__ __forceinline__ uint32_t max_over_group(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));                        // lanes 1 0 3 2 of every four
    if constexpr (GROUP == 4) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false));   // 2 3 0 1
    return x;
}

__device__ __forceinline__ float clamped(float x, float most) { return x != x ? x : fminf(fmaxf(x, -most), most); }

constexpr uint32_t kInf = 0x7F800000u;

// eight FP4 elements of y / scale, rounded to the nearest, ties to even, the largest where they are beyond it (`scale`: a power of two)
__device__ __forceinline__ uint32_t eight_to_fp4(const float (&y)[8], float scale)
{
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
}

// y as stored; scale: FP4, the block's
template <int FMT> __device__ __forceinline__ u32x4_t quantised(float (&y)[8], uint32_t &scale)
{
    u32x4_t w = {0, 0, 0, 0};
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
        uint32_t top = 0;                                      // magnitudes as integers: NaN above infinity above all numbers
#pragma unroll
        for (int i = 0; i < 8; i++) top = max(top, bits(y[i]) & 0x7FFFFFFFu);
        top = max_over_group<kBlock<FMT> / 8>(top);
        const bool nan = top > kInf;
        if constexpr (FMT == ZC_FMT_FP4_E2M1_MX) {
            // 2^(floor(log2 of the largest) - 2); an infinity counts as the largest number
            const int32_t e = (int32_t)min(top >> 23, 254u) - 2;
            scale = nan ? 255u : (uint32_t)max(e, 0);
            w[0] = nan ? 0u : eight_to_fp4(y, block_scale<FMT>(scale));
        } else {
            const float largest = fminf(__uint_as_float(top), 6.0f * 448.0f);
            scale = nan ? 0x7Fu : (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(largest / 6.0f, 0.0f, 0, false) & 0xFFu;
            const float s = block_scale<FMT>(scale);
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = s == 0.0f ? 0.0f : y[i] / s;
            w[0] = nan ? 0u : eight_to_fp4(y, 1.0f);
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

// Every element is divided by the scale of its sequence and head (0: all become 0), rounded to the nearest, ties to even, the largest number where it is
// beyond that.  NaN stays one; in an FP4 block it makes the block's scale NaN.
template <int FMT, int D>
__global__ __launch_bounds__(256) void k_kv_write(RowsDev r)
{
    const uint32_t head = blockIdx.x % r.c.heads, sub = threadIdx.x % kLanes<D>;
    const int32_t token = (int32_t)(blockIdx.x / r.c.heads * kTokens<D> + threadIdx.x / kLanes<D>);
    const uint64_t t = (uint64_t)min(token, (int32_t)r.n_tokens - 1);
    u32x4_t x[2];
    x[0] = *reinterpret_cast<const u32x4_t *>(r.k + t * r.k_token_stride + (uint64_t)head * r.k_head_stride + sub * 8);
    x[1] = *reinterpret_cast<const u32x4_t *>(r.v + t * r.v_token_stride + (uint64_t)head * r.v_head_stride + sub * 8);
    const Place p = place_of<D>(r, head, token);
#pragma unroll
    for (int kv = 0; kv < 2; kv++) {
        const float *scales = kv ? r.c.v_scales : r.c.k_scales;
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            y[2 * i] = __uint_as_float(x[kv][i] << 16);
            y[2 * i + 1] = __uint_as_float(x[kv][i] & 0xFFFF0000u);
        }
        if (scales) {
            const float s = scales[p.unit];
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = s == 0.0f ? 0.0f : y[i] / s;
        }
        uint32_t scale = 0;
        u32x4_t w = quantised<FMT>(y, scale);
        if constexpr (FMT == ZC_FMT_BF16) {
            if (!scales) w = x[kv];                            // bit for bit
        }
        if (!p.there) continue;
        store_eight<FMT>((kv ? r.v_pages : r.k_pages) + p.row * kRowBytes<FMT, D> + sub * kElemBits<FMT>, w);
        if constexpr (kFp4<FMT>) {
            constexpr uint32_t kGroup = kBlock<FMT> / 8;
            if (sub % kGroup == 0) (kv ? r.v_scale_pages : r.k_scale_pages)[p.row * kRowScales<FMT, D> + sub / kGroup] = (uint8_t)scale;
        }
    }
}

// Element times its block's scale times that of its sequence and head, in 32 bits, rounded to BF16; 0 where the token's page is absent.
template <int FMT, int D>
__global__ __launch_bounds__(256) void k_kv_read(RowsDev r)
{
    const uint32_t head = blockIdx.x % r.c.heads, sub = threadIdx.x % kLanes<D>;
    const int32_t token = (int32_t)(blockIdx.x / r.c.heads * kTokens<D> + threadIdx.x / kLanes<D>);
    const Place p = place_of<D>(r, head, token);
    if (!p.ours) return;
    u32x4_t w[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    uint32_t block[2] = {0, 0};
    if (p.there) {
#pragma unroll
        for (int kv = 0; kv < 2; kv++) {
            w[kv] = load_eight<FMT>((kv ? r.c.v : r.c.k) + p.row * kRowBytes<FMT, D> + sub * kElemBits<FMT>);
            if constexpr (kFp4<FMT>) block[kv] = (kv ? r.c.v_blocks : r.c.k_blocks)[p.row * kRowScales<FMT, D> + sub / (kBlock<FMT> / 8)];
        }
    }
#pragma unroll
    for (int kv = 0; kv < 2; kv++) {
        const float *scales = kv ? r.c.v_scales : r.c.k_scales;
        const float s = scales && p.there ? scales[p.unit] : 1.0f;
        float y[8];
        if constexpr (FMT == ZC_FMT_BF16) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                y[2 * i] = __uint_as_float(w[kv][i] << 16);
                y[2 * i + 1] = __uint_as_float(w[kv][i] & 0xFFFF0000u);
            }
        } else if constexpr (!kFp4<FMT>) {
            const u32x4_t b = eight_to_bf16<FMT>(w[kv][0], w[kv][1]);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                y[2 * i] = __uint_as_float(b[i] << 16);
                y[2 * i + 1] = __uint_as_float(b[i] & 0xFFFF0000u);
            }
        } else {
            const u32x4_t b = eight_fp4_to_bf16<FMT>(w[kv][0], block_scale<FMT>(block[kv]));
#pragma unroll
            for (int i = 0; i < 4; i++) {
                y[2 * i] = __uint_as_float(b[i] << 16);
                y[2 * i + 1] = __uint_as_float(b[i] & 0xFFFF0000u);
            }
        }
        u32x4_t out;
#pragma unroll
        for (int i = 0; i < 4; i++) out[i] = pack_bf16(y[2 * i] * s, y[2 * i + 1] * s);
        if constexpr (FMT == ZC_FMT_BF16) {
            if (!scales) out = w[kv];
        }
        uint16_t *to = kv ? r.v + (uint64_t)token * r.v_token_stride + (uint64_t)head * r.v_head_stride : r.k + (uint64_t)token * r.k_token_stride + (uint64_t)head * r.k_head_stride;
        *reinterpret_cast<u32x4_t *>(to + sub * 8) = out;
    }
}

template <int FMT, int D, bool WRITE> int launch(const RowsDev &r, hipStream_t s)
{
    const dim3 blocks((r.n_tokens + kTokens<D> - 1) / kTokens<D> * r.c.heads);
    if constexpr (WRITE) hipLaunchKernelGGL((k_kv_write<FMT, D>), blocks, dim3(256), 0, s, r);
    else hipLaunchKernelGGL((k_kv_read<FMT, D>), blocks, dim3(256), 0, s, r);
    return (int)hipGetLastError();
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
