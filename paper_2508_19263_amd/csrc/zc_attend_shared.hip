// k_attend_shared: both passes of a batch under one prefix in one launch.  The first workgroups take parts of the prefix for rows of
// all sequences (as k_attend_many, or k_attend_few where these are at most 64), those behind them the sequences' own caches (as
// k_attend_few), which fill the places that the former leave.  Replayed from a graph, one pass after the other against one launch: 64 answers
// (8 K/V heads of 128, 4 query heads to each, FP8) of 16 to 777 tokens under 32,768, 76 against 72 - 75 us; five answers (BF16) under 1,531,
// 19.2 against 12.9.  Under a kernel trace 59 us of the former are this kernel's, 590 TFLOP/s, bound like k_attend_many but with tiles
// converted for only two row blocks, and 9 the join of 33 slots; of the latter, 11 and 4, bound by latency.  64 answers over MXFP4 pages 62 - 67 us,
// NVFP4 68.
#include "zc_attend_few.h"
#include "zc_attend_many.h"

namespace zc {

namespace {

// PRE_MANY: the prefix as in k_attend_many, else in k_attend_few with QT
template <int FMT, int D, bool PRE_MANY, int QT>
__global__ __launch_bounds__(256, 2) void k_attend_shared(AttendDev pre, AttendDev own, uint32_t pre_blocks)
{
    constexpr size_t kBytes = PRE_MANY && sizeof(ManyTile<D>) > sizeof(FewShared<D, QT>) ? sizeof(ManyTile<D>) : sizeof(FewShared<D, QT>);
    __shared__ __align__(1024) uint8_t room[kBytes];
    // (A reference to one of the two arguments, chosen here, would have the compiler copy both to scratch memory.)
    if (blockIdx.x < pre_blocks) {
        const uint32_t units = pre.c.heads, id = blockIdx.x / units;
        if constexpr (PRE_MANY) {
            __shared__ ManyTile<D> tile1;
            __shared__ ManyNotes notes;
            attend_many<FMT, D>(pre, blockIdx.x, *reinterpret_cast<ManyTile<D> *>(room), tile1, notes);
        }
        else attend_few<FMT, D, QT, false, false>(pre, blockIdx.x % units, id % pre.splits, id / pre.splits, *reinterpret_cast<FewShared<D, QT> *>(room));
    } else {
        const uint32_t units = own.n_seqs * own.c.heads, id = (blockIdx.x - pre_blocks) / units;
        attend_few<FMT, D, QT, false, false>(own, (blockIdx.x - pre_blocks) % units, id % own.splits, id / own.splits, *reinterpret_cast<FewShared<D, QT> *>(room));
    }
}

template <int FMT, int D> int launch(const AttendDev &pre, const AttendDev &own, uint32_t pre_blocks, uint32_t blocks, bool pre_many, uint32_t tiles, hipStream_t s)
{
    if (pre_many && tiles == 1) hipLaunchKernelGGL((k_attend_shared<FMT, D, true, 1>), dim3(blocks), dim3(256), 0, s, pre, own, pre_blocks);
    else if (pre_many) hipLaunchKernelGGL((k_attend_shared<FMT, D, true, 2>), dim3(blocks), dim3(256), 0, s, pre, own, pre_blocks);
    else if (tiles == 1) hipLaunchKernelGGL((k_attend_shared<FMT, D, false, 1>), dim3(blocks), dim3(256), 0, s, pre, own, pre_blocks);
    else hipLaunchKernelGGL((k_attend_shared<FMT, D, false, 2>), dim3(blocks), dim3(256), 0, s, pre, own, pre_blocks);
    return (int)hipGetLastError();
}
template <int FMT> int launch(const AttendDev &pre, const AttendDev &own, uint32_t head_dim, uint32_t pre_blocks, uint32_t blocks, bool pre_many, uint32_t tiles, hipStream_t s)
{
    return head_dim == 64 ? launch<FMT, 64>(pre, own, pre_blocks, blocks, pre_many, tiles, s) : launch<FMT, 128>(pre, own, pre_blocks, blocks, pre_many, tiles, s);
}

}  // namespace

int launch_attend_shared(const AttendDev &pre, const AttendDev &own, uint32_t format, uint32_t head_dim, bool pre_many, uint32_t tiles, void *stream)
{
    const uint32_t pre_blocks = pre.c.heads * pre.row_blocks * pre.splits, blocks = pre_blocks + own.n_seqs * own.c.heads * own.row_blocks * own.splits;
    const hipStream_t s = (hipStream_t)stream;
    if (format == ZC_FMT_BF16) return launch<ZC_FMT_BF16>(pre, own, head_dim, pre_blocks, blocks, pre_many, tiles, s);
    if (format == ZC_FMT_FP8_E4M3) return launch<ZC_FMT_FP8_E4M3>(pre, own, head_dim, pre_blocks, blocks, pre_many, tiles, s);
    if (format == ZC_FMT_FP8_E5M2) return launch<ZC_FMT_FP8_E5M2>(pre, own, head_dim, pre_blocks, blocks, pre_many, tiles, s);
    if (format == ZC_FMT_FP4_E2M1_MX) return launch<ZC_FMT_FP4_E2M1_MX>(pre, own, head_dim, pre_blocks, blocks, pre_many, tiles, s);
    return launch<ZC_FMT_FP4_E2M1_NV>(pre, own, head_dim, pre_blocks, blocks, pre_many, tiles, s);
}

}  // namespace zc
