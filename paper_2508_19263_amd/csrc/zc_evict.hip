// Eviction from a paged K/V cache by accumulated attention weight: k_evict_select decides which tokens stay, k_evict_move
// brings their keys, values and weights to the pages of another table.
#include <hip/hip_runtime.h>

#include "zc_attend.h"

namespace zc {

namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kThreads = 1024, kGroupWaves = kThreads / 64;
constexpr uint32_t kBins = 2048, kCopies = 8, kRoom = 1024;      // bins of the histogram, its copies, keys of the threshold's bin per wavefront

// Order of the weights as unsigned integers: NaN lowest, -0 equal to +0.  0 is no weight's.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (!(w == w)) return 1;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Inclusive sums over the lanes of a wavefront.
__device__ __forceinline__ uint32_t scan_wave(uint32_t x)
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);      // from one, two, four, eight lanes before, in rows of 16
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);      // the row's sum before, the half's
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);
    return x;
}

// Sum of the 16 numbers before the n-th; every lane of the wavefront gets it.
__device__ __forceinline__ uint32_t sum_before(const uint32_t *x, uint32_t n, uint32_t lane)
{
    const uint32_t v = scan_wave(lane < n ? x[lane & (kGroupWaves - 1)] : 0u);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// One workgroup per (sequence, head).  The keep - sinks - recent largest weights of the middle are those above a threshold and
// the first of those equal to it.  Every wavefront has a stretch of tokens, four consecutive ones to a lane:
//   a histogram of the keys' top 11 bits (sign, exponent and two bits of the mantissa) says which bin the threshold is in;
//   the keys of that bin, some percent, are collected in LDS, where 11 and 10 bits more of them are counted;
//   every wavefront knows how many of its tokens stay, so how many stay in front of its own, and writes them in order.
// Three passes over the weights; their instructions are what bounds it, on one compute unit per sequence and head (16 x 8 times 20,011
// to 65,536 tokens 36 us; six passes, with 8 bits of all keys at a time, took 82 instead of 43 us when it was made of three).  Where a
// bin has more keys than there is room for, they are taken from memory again each time.  HELD: the keys of up to so many times 256
// tokens of a wavefront stay in registers instead (0: none): 4 x 8 times 8,192 tokens 15.9 -> 11.6 us, 4 times 17,062 with their
// move 31.8 -> 28.5, 8 times 53,013 80 -> 73.  The histogram has eight copies for eight neighbouring lanes: weights have few exponents.
template <int HELD>
__global__ __launch_bounds__(kThreads) void k_evict_select(EvictDev e)
{
    __shared__ __align__(16) uint32_t hist[kBins * kCopies];
    __shared__ uint32_t some[kGroupWaves][kRoom];
    __shared__ uint32_t wave_sum[kGroupWaves], wave_more[kGroupWaves];
    __shared__ uint32_t found[2], crowded;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
    for (uint32_t i = tid; i < e.sinks; i += kThreads) kept[i] = (int32_t)i;
    for (uint32_t i = tid; i < e.recent; i += kThreads) kept[e.keep - e.recent + i] = (int32_t)(end + i);
    if (!need) return;
    const uint32_t rounds = (length + kGroupWaves * 256 - 1) / (kGroupWaves * 256), from = wave * rounds * 256;    // the stretch: `rounds` times 256 tokens
    const uint64_t below = (1ull << lane) - 1;

    // f(first token of this lane's four, their keys) for the stretch, four reads on their way at a time; a table's tokens are a
    // multiple of 16, so four from a multiple of 4 that is below the length are inside
    auto key_of = [&](uint32_t r, uint32_t (&key)[4]) {        // 0: not of the middle
        const uint32_t first = from + r * 256 + lane * 4;
        const f32x4u v = *reinterpret_cast<const f32x4u *>(w + min(first, (length - 1) & ~3u));
#pragma unroll
        for (int j = 0; j < 4; j++) key[j] = first + j - begin < end - begin ? weight_key(v[j]) : 0u;
    };
    uint32_t held[HELD ? HELD : 1][4];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int r = 0; r < HELD; r++) key_of((uint32_t)r, held[r]);
    }
    auto over_stretch = [&](auto f) {
        if constexpr (HELD > 0) {
#pragma unroll
            for (uint32_t r = 0; r < HELD; r++)
                if (r < rounds) f(from + r * 256 + lane * 4, held[r]);
        } else {
            for (uint32_t r0 = 0; r0 < rounds; r0 += 4) {
                uint32_t key[4][4];
#pragma unroll
                for (uint32_t k = 0; k < 4; k++) key_of(r0 + k, key[k]);
#pragma unroll
                for (uint32_t k = 0; k < 4; k++)
                    if (r0 + k < rounds) f(from + (r0 + k) * 256 + lane * 4, key[k]);
            }
        }
    };
    auto clear = [&]() {
        for (uint32_t i = tid; i < kBins * kCopies / 4; i += kThreads) reinterpret_cast<uint4 *>(hist)[i] = make_uint4(0, 0, 0, 0);
    };
    // The bin that the need-th largest key is in, given `above` larger keys elsewhere, which becomes how many are larger than that bin.
    auto find = [&](uint32_t &above) {
        uint32_t two[2];                                       // bins 2047 - 2 tid and the one below
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const uint4 *x = reinterpret_cast<const uint4 *>(hist + (kBins - 1 - 2 * tid - k) * kCopies);
            two[k] = (x[0].x + x[0].y + x[0].z + x[0].w) + (x[1].x + x[1].y + x[1].z + x[1].w);
        }
        const uint32_t upto = scan_wave(two[0] + two[1]);
        if (lane == 63) wave_sum[wave] = upto;
        __syncthreads();
        const uint32_t before = above + upto - two[0] - two[1] + sum_before(wave_sum, wave, lane);
        if (before < need && before + two[0] + two[1] >= need) {
            const bool first = before + two[0] >= need;
            found[0] = kBins - 1 - 2 * tid - (first ? 0 : 1);
            found[1] = before + (first ? 0 : two[0]);
        }
        __syncthreads();
        above = found[1];
        return found[0];
    };

    uint32_t above = 0, n_some = 0, n_sure = 0, n_equal = 0;
    clear();
    if (tid == 0) crowded = 0;
    __syncthreads();
    over_stretch([&](uint32_t, const uint32_t (&key)[4]) {
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (key[j]) atomicAdd(&hist[(key[j] >> 21) * kCopies + (lane & (kCopies - 1))], 1u);
    });
    __syncthreads();
    const uint32_t top = find(above);                          // (the middle has more than `need` keys)
    clear();
    // what of the stretch is above the threshold's bin, and the keys of that bin
    over_stretch([&](uint32_t, const uint32_t (&key)[4]) {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            n_sure += key[j] > (top << 21 | 0x1FFFFFu);
            const uint64_t q = __ballot(key[j] >> 21 == top && key[j]);
            if (q) {
                const uint32_t at = n_some + (uint32_t)__popcll(q & below);
                if ((q >> lane & 1) && at < kRoom) some[wave][at] = key[j];
                n_some += (uint32_t)__popcll(q);
            }
        }
    });
    if (n_some > kRoom && lane == 0) crowded = 1;
    __syncthreads();
    const bool in_lds = !crowded;
    // f(key) for the stretch's keys of that bin
    auto over_some = [&](auto f) {
        if (in_lds) {
            for (uint32_t i = lane; i < n_some; i += 64) f(some[wave][i]);
        } else {
            over_stretch([&](uint32_t, const uint32_t (&key)[4]) {
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (key[j] >> 21 == top && key[j]) f(key[j]);
            });
        }
    };
    over_some([&](uint32_t key) { atomicAdd(&hist[(key >> 10 & 2047) * kCopies + (lane & (kCopies - 1))], 1u); });
    __syncthreads();
    uint32_t threshold = top << 11 | find(above);
    clear();
    __syncthreads();
    over_some([&](uint32_t key) { if (key >> 10 == threshold) atomicAdd(&hist[(key & 1023) * kCopies + (lane & (kCopies - 1))], 1u); });
    __syncthreads();
    threshold = threshold << 10 | find(above);
    over_some([&](uint32_t key) { n_sure += key > threshold; n_equal += key == threshold; });
    n_sure = (uint32_t)__builtin_amdgcn_readlane((int)scan_wave(n_sure), 63);
    n_equal = (uint32_t)__builtin_amdgcn_readlane((int)scan_wave(n_equal), 63);
    __syncthreads();                                       // wave_sum is free again
    const uint32_t ties = need - above;
    if (lane == 0) { wave_sum[wave] = n_sure; wave_more[wave] = n_equal; }
    __syncthreads();
    uint32_t sure_before = sum_before(wave_sum, wave, lane), equal_before = sum_before(wave_more, wave, lane);
    over_stretch([&](uint32_t first, const uint32_t (&key)[4]) {
        uint32_t s_in = sure_before, q_in = equal_before;      // of those before this lane's first token
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint64_t s = __ballot(key[j] > threshold);
            s_in += (uint32_t)__popcll(s & below);
            sure_before += (uint32_t)__popcll(s);
        }
        if (__any(key[0] == threshold || key[1] == threshold || key[2] == threshold || key[3] == threshold)) {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint64_t q = __ballot(key[j] == threshold);
                q_in += (uint32_t)__popcll(q & below);
                equal_before += (uint32_t)__popcll(q);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const bool equal = key[j] == threshold;
            const uint32_t at = e.sinks + s_in + min(q_in, ties);
            if ((key[j] > threshold || (equal && q_in < ties)) && at < e.keep) kept[at] = (int32_t)(first + j);
            s_in += key[j] > threshold;
            q_in += equal;
        }
    });
}

template <bool STREAM> __device__ __forceinline__ u32x4 load_piece(const uint8_t *p)
{
    const u32x4 *x = reinterpret_cast<const u32x4 *>(p);
    if constexpr (STREAM) return __builtin_nontemporal_load(x);
    else return *x;
}
template <bool STREAM> __device__ __forceinline__ void store_piece(uint8_t *p, const u32x4 &v)
{
    u32x4 *x = reinterpret_cast<u32x4 *>(p);
    if constexpr (STREAM) __builtin_nontemporal_store(v, x);
    else *x = v;
}

// FP4: a row's block scales, which lie at its number in pools of their own (0 from an absent page)
template <typename T> __device__ __forceinline__ void move_scales_as(const EvictDev &e, bool from_there, uint64_t from, bool to_there, uint64_t to)
{
    const T k = from_there ? reinterpret_cast<const T *>(e.from.k_blocks)[from] : T(0), v = from_there ? reinterpret_cast<const T *>(e.from.v_blocks)[from] : T(0);
    if (!to_there) return;
    reinterpret_cast<T *>(e.k_blocks_to)[to] = k;
    reinterpret_cast<T *>(e.v_blocks_to)[to] = v;
}
__device__ __forceinline__ void move_scales(const EvictDev &e, bool from_there, uint64_t from, bool to_there, uint64_t to)
{
    if (e.row_scales == 8) move_scales_as<uint64_t>(e, from_there, from, to_there, to);
    else if (e.row_scales == 4) move_scales_as<uint32_t>(e, from_there, from, to_there, to);
    else move_scales_as<uint16_t>(e, from_there, from, to_there, to);
}

// 64 rows of keys and of values of one (sequence, head) to a workgroup: where each comes from and goes to is worked out once, then
// every thread has all of its 16-byte pieces (PIECES to a row) on their way before it stores them.  STREAM: past the caches, where a call moves more
// than the memory-side cache holds (1.07 GB: 192 us, 5.6 TB/s, against 215; 67 MB: 13.4 against 11.7 us, 5.7 TB/s).  Bound by reading
// and writing (a copy of contiguous memory reaches 6.2 TB/s).
template <uint32_t PIECES, bool STREAM>
__global__ __launch_bounds__(256) void k_evict_move(EvictDev e, uint32_t blocks_per_head)
{
    constexpr uint32_t kEach = 64 * PIECES < 256 ? 1 : 64 * PIECES / 256;      // pieces per thread (two to a row: of every other thread)
    constexpr uint64_t kNone = ~0ull;
    __shared__ uint64_t src_at[64], dst_at[64];
    const uint32_t unit = blockIdx.x / blocks_per_head, seq = unit / e.from.heads, tid = threadIdx.x;
    const uint32_t count = min((uint32_t)min(max(e.from.lengths[seq], 0), e.from.capacity), e.keep), row0 = blockIdx.x % blocks_per_head * 64;
    if (row0 >= count) return;
    if (tid < 64) {
        uint64_t from = kNone, to = kNone;
        if (row0 + tid < count) {
            const uint32_t dst = row0 + tid, src = (uint32_t)e.kept[(uint64_t)unit * e.keep + dst];
            const int32_t sp = e.from.table[(uint64_t)unit * e.from.table_pages + (src >> e.from.page_shift)];
            const int32_t dp = e.to.table[(uint64_t)unit * e.to.table_pages + (dst >> e.to.page_shift)];
            if ((uint32_t)sp < e.from.n_pages) from = (((uint64_t)sp << e.from.page_shift) + (src & ((1u << e.from.page_shift) - 1))) * (PIECES * 16);
            if (e.row_scales) move_scales(e, (uint32_t)sp < e.from.n_pages, ((uint64_t)(uint32_t)sp << e.from.page_shift) + (src & ((1u << e.from.page_shift) - 1)),
                                          (uint32_t)dp < e.to.n_pages, ((uint64_t)(uint32_t)dp << e.to.page_shift) + (dst & ((1u << e.to.page_shift) - 1)));
            if ((uint32_t)dp < e.to.n_pages) to = (((uint64_t)dp << e.to.page_shift) + (dst & ((1u << e.to.page_shift) - 1))) * (PIECES * 16);
            if (e.weights_to) e.weights_to[(uint64_t)unit * (uint64_t)e.to.capacity + dst] = e.weights[(uint64_t)unit * (uint64_t)e.from.capacity + src];
        }
        src_at[tid] = from;
        dst_at[tid] = to;
    }
    __syncthreads();
    if (PIECES * 64 < 256 && tid >= PIECES * 64) return;
    u32x4 k[kEach], v[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; i++) {
        const uint32_t r = (i * 256 + tid) / PIECES, piece = tid % PIECES;
        const uint64_t from = src_at[r];
        k[i] = v[i] = u32x4{0, 0, 0, 0};                       // a row from an absent page
        if (from != kNone) {
            k[i] = load_piece<STREAM>(e.from.k + from + piece * 16);
            v[i] = load_piece<STREAM>(e.from.v + from + piece * 16);
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < kEach; i++) {
        const uint32_t r = (i * 256 + tid) / PIECES, piece = tid % PIECES;
        const uint64_t to = dst_at[r];
        if (to != kNone) {
            store_piece<STREAM>(e.k_to + to + piece * 16, k[i]);
            store_piece<STREAM>(e.v_to + to + piece * 16, v[i]);
        }
    }
}

template <uint32_t PIECES> void launch_move(const EvictDev &e, uint32_t blocks, uint32_t per_head, bool stream_past, hipStream_t s)
{
    if (stream_past) hipLaunchKernelGGL((k_evict_move<PIECES, true>), dim3(blocks), dim3(256), 0, s, e, per_head);
    else hipLaunchKernelGGL((k_evict_move<PIECES, false>), dim3(blocks), dim3(256), 0, s, e, per_head);
}

}  // namespace

int launch_evict(const EvictDev &e, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    const uint32_t units = e.n_seqs * e.from.heads;
    const uint32_t rounds = ((uint32_t)e.from.capacity + kGroupWaves * 256 - 1) / (kGroupWaves * 256);
    if (rounds <= 2) hipLaunchKernelGGL(k_evict_select<2>, dim3(units), dim3(kThreads), 0, s, e);
    else if (rounds <= 8) hipLaunchKernelGGL(k_evict_select<8>, dim3(units), dim3(kThreads), 0, s, e);
    else if (rounds <= 16) hipLaunchKernelGGL(k_evict_select<16>, dim3(units), dim3(kThreads), 0, s, e);
    else hipLaunchKernelGGL(k_evict_select<0>, dim3(units), dim3(kThreads), 0, s, e);
    int rc = (int)hipGetLastError();
    if (rc) return rc;
    const uint32_t per_head = ((e.keep < (uint32_t)e.from.capacity ? e.keep : (uint32_t)e.from.capacity) + 63) / 64;
    if (!per_head) return 0;
    const bool stream_past = (uint64_t)units * per_head * 64 * e.row_bytes * 4 > kMemorySideCache;       // keys and values, read and written
    if (e.row_bytes == 32) launch_move<2>(e, units * per_head, per_head, stream_past, s);
    else if (e.row_bytes == 64) launch_move<4>(e, units * per_head, per_head, stream_past, s);
    else if (e.row_bytes == 128) launch_move<8>(e, units * per_head, per_head, stream_past, s);
    else launch_move<16>(e, units * per_head, per_head, stream_past, s);
    return (int)hipGetLastError();
}

}  // namespace zc
