// k_attend_few: attention over K/V pages for few query rows (zc_attend_few.h).
#include "zc_attend_few.h"

namespace zc {

namespace {

enum Pages { kThrough, kPast, kChoose };       // the caches; kChoose: as past_caches says

template <int FMT, int D, int QT, bool LOGITS, Pages PAGES>
__global__ __launch_bounds__(kWaves * 64, 2) void k_attend_few(AttendDev a)
{
    __shared__ FewShared<D, QT> shared;
    // Each part begins with another unit: workgroups that lie a round apart go to the same compute unit, where the parts of a long
    // cache would meet (one FP8 cache of 131,072 tokens and 31 of 1,000: 168 -> 128 us, six of 100 to 3,001 13.6 -> 12.4 us).
    const uint32_t unit = (blockIdx.x + blockIdx.y * 13) % gridDim.x;
    if constexpr (PAGES == kChoose) {
        if (past_caches(a, unit, blockIdx.y)) {
            attend_few<FMT, D, QT, LOGITS, true>(a, unit, blockIdx.y, blockIdx.z, shared);
            return;
        }
    }
    attend_few<FMT, D, QT, LOGITS, PAGES == kPast>(a, unit, blockIdx.y, blockIdx.z, shared);
}

// Short FP4 caches, one part and up to 16 rows each, few enough for a compute unit to each: eight wavefronts, every one an eighth of the steps (one cache
// of 640 tokens 7.5 -> 7.0 us, 32 of 2,048 18.1 -> 15.6; bound by the latency of lengths, page numbers and rows, one after the other).
template <int FMT, int D>
__global__ __launch_bounds__(512, 2) void k_attend_short(AttendDev a)
{
    __shared__ FewShared<D, 1, 8> shared;
    attend_few<FMT, D, 1, false, false, 8>(a, blockIdx.x, blockIdx.y, blockIdx.z, shared);
}

template <int FMT, int D, int QT, bool LOGITS> void launch_of(const AttendDev &a, dim3 blocks, hipStream_t s)
{
    if constexpr (kRowBytes<FMT, D> >= kLeastPast) {
        if (a.past_caches) {
            hipLaunchKernelGGL((k_attend_few<FMT, D, QT, LOGITS, kFp4<FMT> ? kPast : kChoose>), blocks, dim3(kWaves * 64), 0, s, a);
            return;
        }
    }
    hipLaunchKernelGGL((k_attend_few<FMT, D, QT, LOGITS, kThrough>), blocks, dim3(kWaves * 64), 0, s, a);
}
template <int FMT, int D> int launch(const AttendDev &a, uint32_t tiles, dim3 blocks, hipStream_t s)
{
    if constexpr (kFp4<FMT>) {
        if (a.eight) {
            hipLaunchKernelGGL((k_attend_short<FMT, D>), blocks, dim3(512), 0, s, a);
            return (int)hipGetLastError();
        }
    }
    if (a.logits && tiles == 1) launch_of<FMT, D, 1, true>(a, blocks, s);
    else if (a.logits) launch_of<FMT, D, 2, true>(a, blocks, s);
    else if (tiles == 1) launch_of<FMT, D, 1, false>(a, blocks, s);
    else launch_of<FMT, D, 2, false>(a, blocks, s);
    return (int)hipGetLastError();
}
template <int FMT> int launch(const AttendDev &a, uint32_t head_dim, uint32_t tiles, dim3 blocks, hipStream_t s)
{
    return head_dim == 64 ? launch<FMT, 64>(a, tiles, blocks, s) : launch<FMT, 128>(a, tiles, blocks, s);
}

}  // namespace

int launch_attend_few(const AttendDev &a, uint32_t format, uint32_t head_dim, uint32_t tiles, void *stream)
{
    const dim3 blocks((a.shared ? 1 : a.n_seqs) * a.c.heads, a.splits, a.row_blocks);
    const hipStream_t s = (hipStream_t)stream;
    if (format == ZC_FMT_BF16) return launch<ZC_FMT_BF16>(a, head_dim, tiles, blocks, s);
    if (format == ZC_FMT_FP8_E4M3) return launch<ZC_FMT_FP8_E4M3>(a, head_dim, tiles, blocks, s);
    if (format == ZC_FMT_FP8_E5M2) return launch<ZC_FMT_FP8_E5M2>(a, head_dim, tiles, blocks, s);
    if (format == ZC_FMT_FP4_E2M1_MX) return launch<ZC_FMT_FP4_E2M1_MX>(a, head_dim, tiles, blocks, s);
    return launch<ZC_FMT_FP4_E2M1_NV>(a, head_dim, tiles, blocks, s);
}

}  // namespace zc
