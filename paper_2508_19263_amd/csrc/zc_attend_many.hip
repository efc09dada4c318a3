// k_attend_many: attention over K/V pages for many query rows (zc_attend_many.h).
#include "zc_attend_many.h"

namespace zc {

namespace {

template <int FMT, int D>
__global__ __launch_bounds__(kManyWaves * 64, 2) void k_attend_many(AttendDev a)
{
    __shared__ ManyTile<D> tile0, tile1;
    __shared__ ManyNotes notes;
    attend_many<FMT, D>(a, blockIdx.x, tile0, tile1, notes);
}

template <int FMT, int D> int launch(const AttendDev &a, uint32_t blocks, hipStream_t s)
{
    hipLaunchKernelGGL((k_attend_many<FMT, D>), dim3(blocks), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}
template <int FMT> int launch(const AttendDev &a, uint32_t head_dim, uint32_t blocks, hipStream_t s)
{
    return head_dim == 64 ? launch<FMT, 64>(a, blocks, s) : launch<FMT, 128>(a, blocks, s);
}

}  // namespace

int launch_attend_many(const AttendDev &a, uint32_t format, uint32_t head_dim, void *stream)
{
    const uint32_t blocks = (a.shared ? 1 : a.n_seqs) * a.c.heads * a.row_blocks * a.splits;
    const hipStream_t s = (hipStream_t)stream;
    if (format == ZC_FMT_BF16) return launch<ZC_FMT_BF16>(a, head_dim, blocks, s);
    if (format == ZC_FMT_FP8_E4M3) return launch<ZC_FMT_FP8_E4M3>(a, head_dim, blocks, s);
    return launch<ZC_FMT_FP8_E5M2>(a, head_dim, blocks, s);
}

}  // namespace zc
