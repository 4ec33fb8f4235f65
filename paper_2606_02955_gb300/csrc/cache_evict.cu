// cache_evict.cu -- fdllm_cache_evict: the heaviest keys of each sequence and head, copied in
// slot order into other pages of the 4-bit prefix cache.
#include <cuda_runtime.h>

#include "cache.cuh"

namespace fdllm {
namespace {

struct EvictArgs {
    CacheView c;
    const int32_t *table;
    int max_pages;
    const int32_t *lens;
    const float *weights;   // [B, heads, max_len]
    int max_len;
    int budget;
    int first;
    int last;
    const int32_t *dst;     // [B, dst_pages]
    int dst_pages;
    int32_t *out_lens;      // [B]
    float *out_weights;     // [B, heads, budget]
    int32_t *out_index;     // [B, heads, budget]
};

// A sequence's cached length, or -1 where it is out of range.
__device__ __forceinline__ int valid_len(const EvictArgs &a, int b)
{
    const int n = a.lens[b];
    return n >= 0 && n <= a.max_len && n <= (a.max_pages << a.c.page_shift) ? n : -1;
}

// Weights as integers in the same order; -0 equals 0, and a NaN comes before everything.
__device__ __forceinline__ uint32_t order_key(float w)
{
    if (w != w)
        return 0u;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// ---- Selection.  One CTA to a sequence and head; the weight of the last key to be kept comes from
// a bisection of the 32-bit order keys: how many keys are at least a candidate, from the highest
// bit in which the keys differ down, until the count is the wanted one or the bits are used up.
// The keys stay in registers (kPerThread a thread, neighbouring slots), so a round costs its
// comparisons and two barriers; a histogram by digits took 32 K atomics on the few bins that
// weights of one magnitude share (72 us for 16 heads of 32000 keys).  A scan of the counts of keys
// above the threshold and at it then places the kept slots in order.  Only counts are shared:
// the result does not depend on any order of arrival.
template <int kThreads>
struct SelectShared {
    int warp_a[32], warp_b[32];
    uint32_t low[32], high[32];
};

// Sum over the CTA, for all threads.
template <int kThreads>
__device__ __forceinline__ int block_sum(int x, SelectShared<kThreads> &sh)
{
    x = __reduce_add_sync(0xFFFFFFFFu, x);
    __syncthreads();  // the sum before is read
    if ((threadIdx.x & 31) == 0)
        sh.warp_a[threadIdx.x >> 5] = x;
    __syncthreads();
    int t = 0;
    const int lane = threadIdx.x & 31;
    if (lane < kThreads / 32)
        t = sh.warp_a[lane];
    return __reduce_add_sync(0xFFFFFFFFu, t);
}

// Keys of a pass: kPerThread neighbouring slots of this thread, from slot `from` on, that compete
// (others count as absent).
template <int kPerThread>
__device__ __forceinline__ void load_keys(const float *w, int from, int lo, int hi,
                                          uint32_t (&key)[kPerThread])
{
#pragma unroll
    for (int e = 0; e < kPerThread; ++e) {
        const int j = from + e;
        key[e] = j >= lo && j < hi ? order_key(w[j]) : 0u;
    }
}

// kThreads * kPerThread slots a pass; a longer row takes several, its keys loaded anew each time.
template <int kThreads, int kPerThread>
__global__ void __launch_bounds__(kThreads) evict_select_kernel(const __grid_constant__ EvictArgs a)
{
    constexpr int kSpan = kThreads * kPerThread;
    __shared__ SelectShared<kThreads> sh;
    pdl_wait();
    const int h = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = (int64_t)b * a.c.heads + h;
    const float *w = a.weights + row * a.max_len;
    int32_t *index = a.out_index + row * a.budget;
    float *kept_w = a.out_weights + row * a.budget;
    const int n = valid_len(a, b);
    const int kept = min(n, a.budget);
    if (h == 0 && threadIdx.x == 0)
        a.out_lens[b] = kept;
    const int lo = min(a.first, max(n, 0)), hi = max(n - a.last, lo);  // the slots that compete
    const bool all = n <= a.budget;
    const int want = a.budget - a.first - a.last;
    const int passes = (max(n, 0) + kSpan - 1) / kSpan;
    uint32_t key[kPerThread];
    uint32_t threshold = 0xFFFFFFFFu;  // keys above it are kept, and `ties` of those equal to it
    int ties = 0;
    if (!all && want > 0) {
        uint32_t low = 0xFFFFFFFFu, high = 0;
        for (int p = 0; p < passes; ++p) {
            const int from = p * kSpan + threadIdx.x * kPerThread;
            load_keys<kPerThread>(w, from, lo, hi, key);
#pragma unroll
            for (int e = 0; e < kPerThread; ++e)
                if (from + e >= lo && from + e < hi) {
                    low = min(low, key[e]);
                    high = max(high, key[e]);
                }
        }
        low = __reduce_min_sync(0xFFFFFFFFu, low);
        high = __reduce_max_sync(0xFFFFFFFFu, high);
        if (lane == 0) {
            sh.low[warp] = low;
            sh.high[warp] = high;
        }
        __syncthreads();
        low = __reduce_min_sync(0xFFFFFFFFu, lane < kThreads / 32 ? sh.low[lane] : 0xFFFFFFFFu);
        high = __reduce_max_sync(0xFFFFFFFFu, lane < kThreads / 32 ? sh.high[lane] : 0u);
        // The largest value that at least `want` keys reach.  `above`: keys known to exceed all
        // values that still come into question.
        const int top = low == high ? -1 : 31 - __clz(low ^ high);
        uint32_t prefix = top < 0 ? low : low & ~((2u << top) - 1u);
        int reach = hi - lo;  // keys of at least `prefix`
        for (int bit = top; bit >= 0 && reach > want; --bit) {
            const uint32_t candidate = prefix | (1u << bit);
            int count = 0;
            for (int p = 0; p < passes; ++p) {
                const int from = p * kSpan + threadIdx.x * kPerThread;
                if (passes > 1)
                    load_keys<kPerThread>(w, from, lo, hi, key);
#pragma unroll
                for (int e = 0; e < kPerThread; ++e)
                    count += key[e] >= candidate && from + e >= lo && from + e < hi ? 1 : 0;
            }
            count = block_sum<kThreads>(count, sh);
            if (count >= want) {
                prefix = candidate;
                reach = count;
            }
        }
        // Either exactly `want` keys reach the prefix, all of them kept, or it is the threshold
        // and some keys equal to it are.
        int over = 0;
        for (int p = 0; p < passes; ++p) {
            const int from = p * kSpan + threadIdx.x * kPerThread;
            if (passes > 1)
                load_keys<kPerThread>(w, from, lo, hi, key);
#pragma unroll
            for (int e = 0; e < kPerThread; ++e)
                over += key[e] > prefix && from + e >= lo && from + e < hi ? 1 : 0;
        }
        over = block_sum<kThreads>(over, sh);
        threshold = prefix;
        if (reach == want) {
            if (prefix == 0)
                ties = want - over;
            else
                threshold = prefix - 1;  // (equal keys among those that reach it: all kept)
        } else {
            ties = want - over;
        }
    }
    int out = 0, seen = 0;
    for (int p = 0; p < passes; ++p) {
        const int from = p * kSpan + threadIdx.x * kPerThread;
        uint32_t sure = 0, tie = 0;  // by slot of this thread
        float x[kPerThread];
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            const int j = from + e;
            x[e] = j < n ? w[j] : 0.0f;
            const uint32_t k = order_key(x[e]);
            const bool competes = j >= lo && j < hi;
            if (j < n && (all || !competes || (want > 0 && k > threshold)))
                sure |= 1u << e;
            else if (j < n && want > 0 && k == threshold)
                tie |= 1u << e;
        }
        // Places: kept before this thread's slots are the sure ones and the first `ties` ties.
        const int mine_s = __popc(sure), mine_t = __popc(tie);
        int upto_s = mine_s, upto_t = mine_t;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const int us = __shfl_up_sync(0xFFFFFFFFu, upto_s, m);
            const int ut = __shfl_up_sync(0xFFFFFFFFu, upto_t, m);
            upto_s += lane >= m ? us : 0;
            upto_t += lane >= m ? ut : 0;
        }
        __syncthreads();
        if (lane == 31) {
            sh.warp_a[warp] = upto_s;
            sh.warp_b[warp] = upto_t;
        }
        __syncthreads();
        int before_s = 0, before_t = 0, total_s = 0, total_t = 0;
        for (int i = 0; i < kThreads / 32; ++i) {
            before_s += i < warp ? sh.warp_a[i] : 0;
            before_t += i < warp ? sh.warp_b[i] : 0;
            total_s += sh.warp_a[i];
            total_t += sh.warp_b[i];
        }
        int t = seen + before_t + upto_t - mine_t;
        int at = out + before_s + upto_s - mine_s + min(t, ties);
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            bool keep = (sure >> e) & 1u;
            if ((tie >> e) & 1u)
                keep = t++ < ties;
            if (keep) {
                index[at] = from + e;
                kept_w[at] = x[e];
                ++at;
            }
        }
        out += total_s;
        seen += total_t;
    }
    for (int j = max(kept, 0) + threadIdx.x; j < a.budget; j += kThreads) {
        index[j] = -1;
        kept_w[j] = 0.0f;
    }
}

// Rows of up to 2048 slots take 256 threads of 8 slots; longer ones 1024 of 32, whose 32768 slots
// stay in registers (rows beyond that are read again each round).
constexpr int kShortRow = 2048;

constexpr int kMoveSlots = 32;

// ---- Moving.  One CTA takes kMoveSlots kept rows of one head: keys as 16-byte pieces; values
// channel by channel, thread d reading the 16-byte pieces (32 slots) of channel d that hold kept
// slots, kBatch of them in flight, and picking the nibbles.  The slots are the same for all
// threads, so every branch is uniform.
constexpr int kBatch = 4;

template <int D>
__global__ void __launch_bounds__(128) evict_move_kernel(const __grid_constant__ EvictArgs a)
{
    __shared__ int64_t src_row[kMoveSlots];    // slot_index of the source, -1: none
    __shared__ int64_t piece_at[kMoveSlots];   // v_byte of a piece's channel 0, -1: none
    __shared__ uint32_t piece_of[kMoveSlots];  // a slot's piece (low half), its place in it
    __shared__ int pieces;
    pdl_wait();
    const int h = blockIdx.y, b = blockIdx.z;
    const int n = valid_len(a, b);
    const int kept = min(n, a.budget);
    const int slot0 = blockIdx.x * kMoveSlots;
    if (slot0 >= kept)
        return;
    const int dpg = page_of(a.c, a.dst, a.dst_pages, b, slot0);
    if (dpg < 0)
        return;
    if (threadIdx.x < kMoveSlots) {
        const int lane = threadIdx.x, j = slot0 + lane;
        int64_t r = -1, v = -1;
        int s = -1;
        if (j < kept) {
            s = a.out_index[((int64_t)b * a.c.heads + h) * a.budget + j];
            const int pg = page_of(a.c, a.table, a.max_pages, b, s);
            if (pg >= 0) {
                r = slot_index(a.c, pg, h, s);
                v = v_byte(a.c, pg, h, 0, s & ~31);
            }
        }
        // kept slots ascend: a piece begins where the 32-slot group changes
        const int before = __shfl_up_sync(0xFFFFFFFFu, s >> 5, 1);
        const uint32_t begins = __ballot_sync(0xFFFFFFFFu, lane == 0 || before != s >> 5);
        const int piece = __popc(begins & ((2u << lane) - 1u)) - 1;
        src_row[lane] = r;
        piece_of[lane] = (uint32_t)piece | ((uint32_t)(s & 31) << 16);
        if ((begins >> lane) & 1u)
            piece_at[piece] = v;
        if (lane == 0)
            pieces = __popc(begins);
    }
    __syncthreads();
    constexpr int kVecs = D / 32;  // 16-byte pieces of a row of key codes
#pragma unroll
    for (int i = threadIdx.x; i < kMoveSlots * kVecs; i += 128) {
        const int j = i / kVecs, p = i % kVecs;
        if (src_row[j] >= 0)
            *reinterpret_cast<uint4 *>(a.c.kc + slot_index(a.c, dpg, h, slot0 + j) * (D / 2) +
                                       16 * p) =
                *reinterpret_cast<const uint4 *>(a.c.kc + src_row[j] * (D / 2) + 16 * p);
    }
    if (threadIdx.x < kMoveSlots && src_row[threadIdx.x] >= 0) {
        const int64_t to = slot_index(a.c, dpg, h, slot0 + threadIdx.x);
        a.c.ka[to] = a.c.ka[src_row[threadIdx.x]];
        a.c.va[to] = a.c.va[src_row[threadIdx.x]];
    }
    const int d = threadIdx.x;
    if (D < 128 && d >= D)
        return;
    const int64_t step = (int64_t)d << (a.c.page_shift - 1);
    uint32_t out[kMoveSlots / 8];
    uint4 x[kBatch];
    int batch = -kBatch;  // the first piece in x
#pragma unroll
    for (int q = 0; q < kMoveSlots / 8; ++q) {
        uint32_t word = 0;
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const uint32_t f = piece_of[8 * q + e];
            const int piece = (int)(f & 0xFFFFu), in = (int)(f >> 16);
            if (piece >= batch + kBatch) {
                batch = piece;
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    x[i] = make_uint4(0, 0, 0, 0);
                    if (batch + i < pieces && piece_at[batch + i] >= 0)
                        x[i] = *reinterpret_cast<const uint4 *>(a.c.vc + piece_at[batch + i] + step);
                }
            }
            uint4 y = x[0];
#pragma unroll
            for (int i = 1; i < kBatch; ++i)
                if (piece - batch == i)
                    y = x[i];
            const uint32_t lo = (in & 8) ? y.y : y.x, hi = (in & 8) ? y.w : y.z;
            word |= ((((in & 16) ? hi : lo) >> (4 * (in & 7))) & 15u) << (4 * e);
        }
        out[q] = word;
    }
    *reinterpret_cast<uint4 *>(a.c.vc + v_byte(a.c, dpg, h, d, slot0)) =
        make_uint4(out[0], out[1], out[2], out[3]);
}

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" fdllm_status fdllm_cache_evict(const fdllm_cache *cache, const int32_t *block_table,
                                          int B, int max_pages, const int32_t *cache_lens,
                                          const float *weights, int max_len, int budget,
                                          int keep_first, int keep_last,
                                          const int32_t *dst_table, int dst_max_pages,
                                          int32_t *out_lens, float *out_weights,
                                          int32_t *out_index, void *stream)
{
    EvictArgs a = {};
    const fdllm_status st = check_cache(cache, a.c);
    if (st != FDLLM_OK)
        return st;
    if (!check_table(block_table, B, max_pages, a.c.page_shift, a.c.heads) ||
        !check_table(dst_table, B, dst_max_pages, a.c.page_shift, a.c.heads) || !cache_lens ||
        !weights || max_len < 1 || budget < 1 || keep_first < 0 || keep_last < 0 ||
        (int64_t)keep_first + keep_last > budget ||
        ((int64_t)dst_max_pages << a.c.page_shift) < budget || !out_lens || !out_weights ||
        !out_index)
        return FDLLM_ERR_ARG;
    a.table = block_table;
    a.max_pages = max_pages;
    a.lens = cache_lens;
    a.weights = weights;
    a.max_len = max_len;
    a.budget = budget;
    a.first = keep_first;
    a.last = keep_last;
    a.dst = dst_table;
    a.dst_pages = dst_max_pages;
    a.out_lens = out_lens;
    a.out_weights = out_weights;
    a.out_index = out_index;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool short_rows = max_len <= kShortRow;
    if ((short_rows ? launch(evict_select_kernel<256, 8>, dim3(a.c.heads, B), dim3(256), 0, s, true, a)
                    : launch(evict_select_kernel<1024, 32>, dim3(a.c.heads, B), dim3(1024), 0, s, true,
                             a)) != cudaSuccess)
        return FDLLM_ERR_CUDA;
    const dim3 grid((budget + kMoveSlots - 1) / kMoveSlots, a.c.heads, B);
    const cudaError_t e =
        a.c.D == 128 ? launch(evict_move_kernel<128>, grid, dim3(128), 0, s, true, a)
                     : launch(evict_move_kernel<64>, grid, dim3(128), 0, s, true, a);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}
