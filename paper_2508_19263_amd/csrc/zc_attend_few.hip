// k_attend_few: attention over K/V pages for few query rows (zc_attend_few.h).
#include "zc_attend_few.h"

namespace zc {

namespace {

template <int FMT, int D, int QT, bool LOGITS>
__global__ __launch_bounds__(kWaves * 64, 2) void k_attend_few(AttendDev a)
{
    __shared__ FewShared<D, QT> shared;
    // Each part begins with another unit: workgroups that lie a round apart go to the same compute unit, where the parts of a long
    // cache would meet (one FP8 cache of 131,072 tokens and 31 of 1,000: 168 -> 128 us, six of 100 to 3,001 13.6 -> 12.4 us).
    attend_few<FMT, D, QT, LOGITS>(a, (blockIdx.x + blockIdx.y * 13) % gridDim.x, blockIdx.y, blockIdx.z, shared);
}

template <int FMT, int D> int launch(const AttendDev &a, uint32_t tiles, dim3 blocks, hipStream_t s)
{
    if (a.logits && tiles == 1) hipLaunchKernelGGL((k_attend_few<FMT, D, 1, true>), blocks, dim3(kWaves * 64), 0, s, a);
    else if (a.logits) hipLaunchKernelGGL((k_attend_few<FMT, D, 2, true>), blocks, dim3(kWaves * 64), 0, s, a);
    else if (tiles == 1) hipLaunchKernelGGL((k_attend_few<FMT, D, 1, false>), blocks, dim3(kWaves * 64), 0, s, a);
    else hipLaunchKernelGGL((k_attend_few<FMT, D, 2, false>), blocks, dim3(kWaves * 64), 0, s, a);
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
    return launch<ZC_FMT_FP8_E5M2>(a, head_dim, tiles, blocks, s);
}

}  // namespace zc
