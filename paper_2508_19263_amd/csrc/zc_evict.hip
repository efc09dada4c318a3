// Eviction from a paged K/V cache by accumulated attention weight: k_evict_select decides which tokens stay, k_evict_move
// brings their keys, values and weights to the pages of another table.
#include <hip/hip_runtime.h>

#include "zc_attend.h"

namespace zc {

namespace {

constexpr uint32_t kThreads = 1024, kGroupWaves = kThreads / 64;

// Order of the weights as unsigned integers: NaN lowest, -0 equal to +0.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (!(w == w)) return 0;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// One workgroup per (sequence, head).  The keep - sinks - recent largest weights of the middle are those above a threshold and
// the first of those equal to it; three passes over the weights (11, 11 and 10 bits of the key at a time, a histogram in LDS each)
// find it.  Then every wavefront counts a stretch of its own, and once it knows what lies before it writes its tokens in order.
// Bound by latency: the weights, 4 bytes a token, are read from the L2 after the first pass.
__global__ __launch_bounds__(kThreads) void k_evict_select(EvictDev e)
{
    __shared__ uint32_t hist[2048];
    __shared__ uint32_t wave_sum[kGroupWaves], wave_more[kGroupWaves];
    __shared__ uint32_t found_bin, found_above;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t unit = blockIdx.x, head = unit % e.from.heads, seq = unit / e.from.heads;
    const int32_t length = min(max(e.from.lengths[seq], 0), e.from.capacity);
    int32_t *kept = e.kept + (uint64_t)unit * e.keep;
    const uint32_t count = min((uint32_t)length, e.keep);
    if (head == 0 && tid == 0) e.lengths_to[seq] = (int32_t)count;
    for (uint32_t i = count + tid; i < e.keep; i += kThreads) kept[i] = -1;
    if ((uint32_t)length <= e.keep) {
        for (uint32_t i = tid; i < count; i += kThreads) kept[i] = (int32_t)i;
        return;
    }
    const float *w = e.weights + (uint64_t)unit * (uint64_t)e.from.capacity;
    const uint32_t begin = e.sinks, end = (uint32_t)length - e.recent, need = e.keep - e.sinks - e.recent;   // the middle, of which `need` stay

    // ---- the threshold: `above` keys of the middle are larger, and need - above of those equal to it stay
    uint32_t prefix = 0, mask = 0, above = 0;
    for (int pass = 0; pass < 3; pass++) {
        const uint32_t shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
        for (uint32_t i = tid; i < 2048; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (uint32_t i = begin + tid; i < end; i += kThreads) {
            const uint32_t key = weight_key(w[i]);
            if ((key & mask) == prefix) atomicAdd(&hist[key >> shift & (bins - 1)], 1u);
        }
        __syncthreads();
        // bins from the top: thread t has the two bins 2047 - 2t and 2046 - 2t
        const uint32_t hi = hist[2047 - 2 * tid], lo = hist[2046 - 2 * tid];
        uint32_t sum = hi + lo;
        for (uint32_t d = 1; d < 64; d *= 2) {
            const uint32_t x = __shfl_up(sum, d);
            if (lane >= d) sum += x;
        }
        if (lane == 63) wave_sum[wave] = sum;
        if (tid == 0) found_bin = 0xFFFFFFFFu;
        __syncthreads();
        uint32_t before = above;
        for (uint32_t i = 0; i < wave; i++) before += wave_sum[i];
        before += sum - hi - lo;                           // keys above this thread's bins
        if (before < need && before + hi >= need) { found_bin = 2047 - 2 * tid; found_above = before; }
        else if (before + hi < need && before + hi + lo >= need) { found_bin = 2046 - 2 * tid; found_above = before + hi; }
        __syncthreads();
        if (found_bin == 0xFFFFFFFFu) break;               // need == 0: every key is below the threshold
        prefix |= found_bin << shift;
        mask |= (bins - 1) << shift;
        above = found_above;
        __syncthreads();
    }
    const bool none = need == 0;
    const uint32_t threshold = prefix, ties = need - above;

    // ---- stretches of whole wavefronts: what each holds above the threshold and at it
    const uint32_t per = ((uint32_t)length + kThreads - 1) / kThreads * 64, from = min(wave * per, (uint32_t)length), to = min(from + per, (uint32_t)length);
    uint32_t sure = 0, equal = 0;
    for (uint32_t i = from + lane; i < to; i += 64) {
        const bool middle = i >= begin && i < end;
        const uint32_t key = middle && !none ? weight_key(w[i]) : 0;
        sure += !middle || (!none && key > threshold);
        equal += middle && !none && key == threshold;
    }
    for (uint32_t d = 1; d < 64; d *= 2) { sure += __shfl_xor(sure, d); equal += __shfl_xor(equal, d); }
    if (lane == 0) { wave_sum[wave] = sure; wave_more[wave] = equal; }
    __syncthreads();
    uint32_t sure_before = 0, equal_before = 0;
    for (uint32_t i = 0; i < wave; i++) { sure_before += wave_sum[i]; equal_before += wave_more[i]; }
    const uint64_t below = (1ull << lane) - 1;
    for (uint32_t i0 = from; i0 < to; i0 += 64) {
        const uint32_t i = i0 + lane;
        const bool in = i < to, middle = in && i >= begin && i < end;
        const uint32_t key = middle && !none ? weight_key(w[i]) : 0;
        const bool is_sure = in && (!middle || (!none && key > threshold)), is_equal = middle && !none && key == threshold;
        const uint64_t s = __ballot(is_sure), q = __ballot(is_equal);
        const uint32_t rank = equal_before + (uint32_t)__popcll(q & below);
        const uint32_t at = sure_before + (uint32_t)__popcll(s & below) + min(rank, ties);
        if ((is_sure || (is_equal && rank < ties)) && at < e.keep) kept[at] = (int32_t)i;
        sure_before += (uint32_t)__popcll(s);
        equal_before += (uint32_t)__popcll(q);
    }
}

// 16 bytes of a key's or value's row per thread; a workgroup takes 256 rows of one (sequence, head).  Bound by reading and writing them.
__global__ __launch_bounds__(256) void k_evict_move(EvictDev e, uint32_t blocks_per_head, uint32_t rows_per_block)
{
    __shared__ int32_t index[256];
    const uint32_t unit = blockIdx.x / blocks_per_head, seq = unit / e.from.heads;
    const int32_t length = min(max(e.from.lengths[seq], 0), e.from.capacity);
    const uint32_t count = min((uint32_t)length, e.keep), row0 = blockIdx.x % blocks_per_head * rows_per_block;
    if (row0 >= count) return;
    const uint32_t rows = min(rows_per_block, count - row0), pieces = e.row_bytes / 16;
    if (threadIdx.x < rows) {
        const int32_t i = e.kept[(uint64_t)unit * e.keep + row0 + threadIdx.x];
        index[threadIdx.x] = i;
        if (e.weights_to) e.weights_to[(uint64_t)unit * (uint64_t)e.to.capacity + row0 + threadIdx.x] = e.weights[(uint64_t)unit * (uint64_t)e.from.capacity + (uint32_t)i];
    }
    __syncthreads();
    const int32_t *from_table = e.from.table + (uint64_t)unit * e.from.table_pages, *to_table = e.to.table + (uint64_t)unit * e.to.table_pages;
    for (uint32_t x = threadIdx.x; x < rows * pieces; x += 256) {
        const uint32_t r = x / pieces, piece = x % pieces, src = (uint32_t)index[r], dst = row0 + r;
        const int32_t sp = from_table[src >> e.from.page_shift], dp = to_table[dst >> e.to.page_shift];
        if ((uint32_t)dp >= e.to.n_pages) continue;
        const uint64_t dst_at = (((uint64_t)dp << e.to.page_shift) + (dst & ((1u << e.to.page_shift) - 1))) * e.row_bytes + piece * 16;
        uint4 k = make_uint4(0, 0, 0, 0), v = k;
        if ((uint32_t)sp < e.from.n_pages) {
            const uint64_t src_at = (((uint64_t)sp << e.from.page_shift) + (src & ((1u << e.from.page_shift) - 1))) * e.row_bytes + piece * 16;
            k = *reinterpret_cast<const uint4 *>(e.from.k + src_at);
            v = *reinterpret_cast<const uint4 *>(e.from.v + src_at);
        }
        *reinterpret_cast<uint4 *>(e.k_to + dst_at) = k;
        *reinterpret_cast<uint4 *>(e.v_to + dst_at) = v;
    }
}

}  // namespace

int launch_evict(const EvictDev &e, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    const uint32_t units = e.n_seqs * e.from.heads;
    hipLaunchKernelGGL(k_evict_select, dim3(units), dim3(kThreads), 0, s, e);
    int rc = (int)hipGetLastError();
    if (rc) return rc;
    const uint32_t most = e.keep < (uint32_t)e.from.capacity ? e.keep : (uint32_t)e.from.capacity, rows_per_block = 64;
    const uint32_t per_head = (most + rows_per_block - 1) / rows_per_block;
    if (!per_head) return 0;
    hipLaunchKernelGGL(k_evict_move, dim3(units * per_head), dim3(256), 0, s, e, per_head, rows_per_block);
    return (int)hipGetLastError();
}

}  // namespace zc
