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

constexpr int kSelectThreads = 512;

// Exclusive rank of this thread among the threads whose flag is set, and their number.
__device__ __forceinline__ int block_rank(bool flag, int *warp_counts, int &total)
{
    const uint32_t ballot = __ballot_sync(0xFFFFFFFFu, flag);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();  // the counts of the call before are read
    if (lane == 0)
        warp_counts[warp] = __popc(ballot);
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kSelectThreads / 32; ++w) {
        const int n = warp_counts[w];
        before += w < warp ? n : 0;
        total += n;
    }
    return before + __popc(ballot & ((1u << lane) - 1u));
}

// One CTA to a sequence and head.  The weight of the last key to be kept comes from four passes
// of a radix select over the weights between the protected ends (8 bits a pass, from the top);
// a last pass writes the kept slots in order.  Integer counts: the result does not depend on
// the order of the atomics.
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(
    const __grid_constant__ EvictArgs a)
{
    __shared__ int hist[256];
    __shared__ int warp_counts[kSelectThreads / 32];
    __shared__ uint32_t sh_prefix;
    __shared__ int sh_need;
    pdl_wait();
    const int h = blockIdx.x, b = blockIdx.y;
    const int64_t row = (int64_t)b * a.c.heads + h;
    const float *w = a.weights + row * a.max_len;
    int32_t *index = a.out_index + row * a.budget;
    float *kept_w = a.out_weights + row * a.budget;
    const int n = valid_len(a, b);
    const int kept = min(n, a.budget);
    if (h == 0 && threadIdx.x == 0)
        a.out_lens[b] = kept;
    const int lo = min(a.first, n), hi = max(n - a.last, lo);  // the slots that compete
    uint32_t threshold = 0;
    int ties = 0;
    const bool all = n <= a.budget;
    const int want = a.budget - a.first - a.last;
    if (!all && want > 0) {
        uint32_t prefix = 0;
        int need = want;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += kSelectThreads)
                hist[i] = 0;
            __syncthreads();
            for (int j = lo + threadIdx.x; j < hi; j += kSelectThreads) {
                const uint32_t key = order_key(w[j]);
                if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)))
                    atomicAdd(&hist[(key >> shift) & 255u], 1);
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int bin = 255;
                while (bin > 0 && hist[bin] < need)
                    need -= hist[bin--];
                sh_prefix = prefix | ((uint32_t)bin << shift);
                sh_need = need;
            }
            __syncthreads();
            prefix = sh_prefix;
            need = sh_need;
        }
        threshold = prefix;
        ties = need;
    }
    int out = 0, seen = 0;
    for (int base = 0; base < max(n, 0); base += kSelectThreads) {
        const int j = base + threadIdx.x;
        bool keep = false, tie = false;
        float x = 0.0f;
        if (j < n) {
            x = w[j];
            const uint32_t key = order_key(x);
            const bool competes = j >= lo && j < hi;
            keep = all || !competes || (want > 0 && key > threshold);
            tie = !all && competes && want > 0 && key == threshold;
        }
        int total;
        const int rank = block_rank(tie, warp_counts, total);
        keep = keep || (tie && seen + rank < ties);
        seen += total;
        const int at = out + block_rank(keep, warp_counts, total);
        out += total;
        if (keep) {
            index[at] = j;
            kept_w[at] = x;
        }
    }
    for (int j = max(kept, 0) + threadIdx.x; j < a.budget; j += kSelectThreads) {
        index[j] = -1;
        kept_w[j] = 0.0f;
    }
}

constexpr int kMoveSlots = 32;

// One CTA moves kMoveSlots kept rows of one head: keys as 16-byte pieces, values channel by
// channel (thread d gathers the nibbles of channel d into 16 bytes).
template <int D>
__global__ void __launch_bounds__(128) evict_move_kernel(const __grid_constant__ EvictArgs a)
{
    __shared__ int64_t src_row[kMoveSlots];   // slot_index of the source, -1: none
    __shared__ int64_t src_byte[kMoveSlots];  // v_byte of channel 0
    __shared__ int src_slot[kMoveSlots];
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
        const int j = slot0 + threadIdx.x;
        int64_t r = -1, v = 0;
        int s = 0;
        if (j < kept) {
            s = a.out_index[((int64_t)b * a.c.heads + h) * a.budget + j];
            const int pg = page_of(a.c, a.table, a.max_pages, b, s);
            if (pg >= 0) {
                r = slot_index(a.c, pg, h, s);
                v = v_byte(a.c, pg, h, 0, s);
            }
        }
        src_row[threadIdx.x] = r;
        src_byte[threadIdx.x] = v;
        src_slot[threadIdx.x] = s;
    }
    __syncthreads();
    constexpr int kVecs = D / 32;  // 16-byte pieces of a row of key codes
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
    if (d < D) {
        const int64_t step = (int64_t)d << (a.c.page_shift - 1);
        uint32_t x[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kMoveSlots; ++j) {
            uint32_t code = 0;
            if (src_row[j] >= 0)
                code = (a.c.vc[src_byte[j] + step] >> (4 * (src_slot[j] & 1))) & 15u;
            x[j >> 3] |= code << (4 * (j & 7));
        }
        *reinterpret_cast<uint4 *>(a.c.vc + v_byte(a.c, dpg, h, d, slot0)) =
            make_uint4(x[0], x[1], x[2], x[3]);
    }
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
    if (launch(evict_select_kernel, dim3(a.c.heads, B), dim3(kSelectThreads), 0, s, true, a) !=
        cudaSuccess)
        return FDLLM_ERR_CUDA;
    const dim3 grid((budget + kMoveSlots - 1) / kMoveSlots, a.c.heads, B);
    const cudaError_t e =
        a.c.D == 128 ? launch(evict_move_kernel<128>, grid, dim3(128), 0, s, true, a)
                     : launch(evict_move_kernel<64>, grid, dim3(128), 0, s, true, a);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}
