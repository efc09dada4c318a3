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
// the first of those equal to it.  A wavefront has a stretch of tokens of its own, up to N of them per lane held as keys in
// registers (N = 0: read anew each time).  Four passes over the keys, 8 bits at a time from the top, find the threshold: a histogram in
// LDS has 32 copies, one per lane of half a wavefront, side by side in the banks, so that the few exponents that weights have cost
// no waits (with one copy of 2,048 bins the passes over 65,536 tokens took 100 us).  Then every wavefront counts its stretch, and
// once it knows what lies before it writes its tokens in order.  Bound by latency.
template <int N>
__global__ __launch_bounds__(kThreads) void k_evict_select(EvictDev e)
{
    __shared__ __align__(16) uint32_t hist[256 * 32];
    __shared__ __align__(16) uint32_t total[256];
    __shared__ uint32_t wave_sum[kGroupWaves], wave_more[kGroupWaves];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t unit = blockIdx.x, head = unit % e.from.heads, seq = unit / e.from.heads;
    const uint32_t length = (uint32_t)min(max(e.from.lengths[seq], 0), e.from.capacity);
    int32_t *kept = e.kept + (uint64_t)unit * e.keep;
    const uint32_t count = min(length, e.keep);
    if (head == 0 && tid == 0) e.lengths_to[seq] = (int32_t)count;
    for (uint32_t i = count + tid; i < e.keep; i += kThreads) kept[i] = -1;
    if (length <= e.keep) {
        for (uint32_t i = tid; i < count; i += kThreads) kept[i] = (int32_t)i;
        return;
    }
    const float *w = e.weights + (uint64_t)unit * (uint64_t)e.from.capacity;
    const uint32_t begin = e.sinks, end = length - e.recent, need = e.keep - e.sinks - e.recent;   // the middle, of which `need` stay
    const uint32_t rounds = (length + kThreads - 1) / kThreads, from = wave * rounds * 64;         // the stretch: `rounds` times 64 tokens

    uint32_t keys[N ? N : 1];
    if constexpr (N > 0) {
#pragma unroll
        for (int j = 0; j < N; j++) {
            const uint32_t i = from + (uint32_t)j * 64 + lane;
            float x = 0.0f;
            if ((uint32_t)j < rounds && i >= begin && i < end) x = w[i];
            keys[j] = weight_key(x);
        }
    }
    // f(token, its key, whether it is of the middle) for the stretch, 64 tokens at a time
    auto over_stretch = [&](auto f) {
        if constexpr (N > 0) {
#pragma unroll
            for (int j = 0; j < N; j++)
                if ((uint32_t)j < rounds) {
                    const uint32_t i = from + (uint32_t)j * 64 + lane;
                    f(i, keys[j], i >= begin && i < end);
                }
        } else {
            for (uint32_t j0 = 0; j0 < rounds; j0 += 8) {          // eight reads on their way at a time
                float x[8];
#pragma unroll
                for (uint32_t j = 0; j < 8; j++) {
                    const uint32_t i = from + (j0 + j) * 64 + lane;
                    x[j] = j0 + j < rounds && i >= begin && i < end ? w[i] : 0.0f;
                }
#pragma unroll
                for (uint32_t j = 0; j < 8; j++)
                    if (j0 + j < rounds) {
                        const uint32_t i = from + (j0 + j) * 64 + lane;
                        f(i, weight_key(x[j]), i >= begin && i < end);
                    }
            }
        }
    };

    // ---- the threshold: `above` keys of the middle are larger, and need - above of those equal to it stay
    uint32_t threshold = 0, above = 0;
    if (need) {
        uint32_t mask = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (uint32_t i = tid; i < 256 * 32 / 4; i += kThreads) reinterpret_cast<uint4 *>(hist)[i] = make_uint4(0, 0, 0, 0);
            __syncthreads();
            over_stretch([&](uint32_t, uint32_t key, bool middle) {
                if (middle && (key & mask) == threshold) atomicAdd(&hist[(key >> shift & 255) * 32 + (lane & 31)], 1u);
            });
            __syncthreads();
            {
                const uint4 x = reinterpret_cast<const uint4 *>(hist)[tid * 2], y = reinterpret_cast<const uint4 *>(hist)[tid * 2 + 1];
                uint32_t sum = x.x + x.y + x.z + x.w + y.x + y.y + y.z + y.w;        // a quarter of bin tid / 4
                sum += __shfl_xor(sum, 1);
                sum += __shfl_xor(sum, 2);
                if ((tid & 3) == 0) total[tid / 4] = sum;
            }
            __syncthreads();
            // every wavefront for itself: lane n has bins 255 - 4 n and the three below
            const uint4 bins = reinterpret_cast<const uint4 *>(total)[63 - lane];
            const uint32_t four = bins.x + bins.y + bins.z + bins.w;
            uint32_t upto = four;
            for (uint32_t d = 1; d < 64; d *= 2) {
                const uint32_t x = __shfl_up(upto, d);
                if (lane >= d) upto += x;
            }
            const uint64_t reached = __ballot(above + upto >= need);                 // not 0: the middle has more than `need` keys
            const int who = __ffsll((unsigned long long)reached) - 1;
            uint32_t before = above + upto - four, bin = 255 - 4 * lane;
            if (before + bins.w < need) {
                before += bins.w; bin--;
                if (before + bins.z < need) {
                    before += bins.z; bin--;
                    if (before + bins.y < need) { before += bins.y; bin--; }
                }
            }
            above = __shfl(before, who);
            threshold |= (uint32_t)__shfl(bin, who) << shift;
            mask |= 255u << shift;
        }
    }
    const uint32_t ties = need - above;
    auto sure = [&](uint32_t i, uint32_t key, bool middle) { return i < length && (!middle || (need && key > threshold)); };
    auto equal = [&](uint32_t key, bool middle) { return middle && need && key == threshold; };

    uint32_t n_sure = 0, n_equal = 0;
    over_stretch([&](uint32_t i, uint32_t key, bool middle) {
        n_sure += sure(i, key, middle);
        n_equal += equal(key, middle);
    });
    for (uint32_t d = 1; d < 64; d *= 2) { n_sure += __shfl_xor(n_sure, d); n_equal += __shfl_xor(n_equal, d); }
    if (lane == 0) { wave_sum[wave] = n_sure; wave_more[wave] = n_equal; }
    __syncthreads();
    uint32_t sure_before = 0, equal_before = 0;
    for (uint32_t i = 0; i < wave; i++) { sure_before += wave_sum[i]; equal_before += wave_more[i]; }
    const uint64_t below = (1ull << lane) - 1;
    over_stretch([&](uint32_t i, uint32_t key, bool middle) {
        const bool is_sure = sure(i, key, middle), is_equal = equal(key, middle);
        const uint64_t s = __ballot(is_sure), q = __ballot(is_equal);
        const uint32_t rank = equal_before + (uint32_t)__popcll(q & below);
        const uint32_t at = sure_before + (uint32_t)__popcll(s & below) + min(rank, ties);
        if ((is_sure || (is_equal && rank < ties)) && at < e.keep) kept[at] = (int32_t)i;
        sure_before += (uint32_t)__popcll(s);
        equal_before += (uint32_t)__popcll(q);
    });
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
    const uint32_t rounds = ((uint32_t)e.from.capacity + kThreads - 1) / kThreads;
    if (rounds <= 8) hipLaunchKernelGGL(k_evict_select<8>, dim3(units), dim3(kThreads), 0, s, e);
    else if (rounds <= 16) hipLaunchKernelGGL(k_evict_select<16>, dim3(units), dim3(kThreads), 0, s, e);
    else hipLaunchKernelGGL(k_evict_select<0>, dim3(units), dim3(kThreads), 0, s, e);
    int rc = (int)hipGetLastError();
    if (rc) return rc;
    const uint32_t most = e.keep < (uint32_t)e.from.capacity ? e.keep : (uint32_t)e.from.capacity, rows_per_block = 64;
    const uint32_t per_head = (most + rows_per_block - 1) / rows_per_block;
    if (!per_head) return 0;
    hipLaunchKernelGGL(k_evict_move, dim3(units * per_head), dim3(256), 0, s, e, per_head, rows_per_block);
    return (int)hipGetLastError();
}

}  // namespace zc
