// cache_evict.cu -- fdllm_cache_evict: the heaviest keys of each sequence and head, copied in
// slot order into other pages of the 4-bit prefix cache.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "cache.cuh"

namespace cg = cooperative_groups;

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
// a radix select over the 32-bit order keys, four bits a round from the highest in which the keys
// differ.  The row passes through shared memory once (coalesced in, neighbouring slots to a thread
// out) and its keys stay in registers; a thread counts its digits in one 64-bit number, four bits
// a digit, and a warp adds them up with eight reductions, pass by pass into 32 bits.  (A histogram in shared memory took 32 K
// atomics on the few bins that weights of one magnitude share: 72 us for 16 heads of 32000 keys;
// a bisection by single bits 38 us, mostly its 32 rounds' barriers.)  A scan of the counts of keys
// above the threshold and at it then places the kept slots in order.  Only counts are shared: the
// result does not depend on any order of arrival.
//
// A long row takes a cluster of kCluster CTAs, neighbouring parts of the row by rank: they leave
// their counts in one another's shared memory.
template <int kThreads, int kPerThread, int kCluster>
struct SelectShared {
    int digits[2][kThreads / 32][16];      // counts of the warps, by the round's parity
    int cta_digits[2][kCluster][16];       // of the CTAs
    int sure[32], ties[32];
    int cta_sure[kCluster], cta_ties[kCluster];
    uint32_t low[32], high[32];
    uint32_t cta_low[kCluster], cta_high[kCluster];
    // slots of a pass; a thread's are kPerThread + 1 apart, so that their reads share no bank
    float w[kThreads * (kPerThread + 1)];
};

// A value of this CTA for every CTA of the cluster, at the same place of each one's shared memory.
template <int kCluster, typename V>
__device__ __forceinline__ void tell(V *slots, V value)
{
    if constexpr (kCluster == 1) {
        slots[0] = value;
    } else {
        cg::cluster_group cluster = cg::this_cluster();
        const unsigned rank = cluster.block_rank();
        for (int i = 0; i < kCluster; ++i)
            cluster.map_shared_rank(slots, i)[rank] = value;
    }
}

template <int kCluster>
__device__ __forceinline__ void meet()
{
    if constexpr (kCluster == 1)
        __syncthreads();
    else
        cg::this_cluster().sync();
}

// kCluster * kThreads * kPerThread slots a pass; a longer row takes several, its keys loaded anew
// each time.
template <int kThreads, int kPerThread, int kCluster>
__global__ void __launch_bounds__(kThreads) evict_select_kernel(const __grid_constant__ EvictArgs a)
{
    constexpr int kSpan = kThreads * kPerThread, kWarps = kThreads / 32;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    auto &sh = *reinterpret_cast<SelectShared<kThreads, kPerThread, kCluster> *>(smem_raw);
    pdl_wait();
    if constexpr (kCluster > 1)
        meet<kCluster>();  // every CTA's shared memory is there
    const int rank = kCluster == 1 ? 0 : (int)cg::this_cluster().block_rank();
    const int h = blockIdx.x / kCluster, b = blockIdx.y, lane = threadIdx.x & 31,
              warp = threadIdx.x >> 5;
    const int64_t row = (int64_t)b * a.c.heads + h;
    const float *w = a.weights + row * a.max_len;
    int32_t *index = a.out_index + row * a.budget;
    float *kept_w = a.out_weights + row * a.budget;
    const int n = valid_len(a, b);
    const int kept = min(n, a.budget);
    if (h == 0 && rank == 0 && threadIdx.x == 0)
        a.out_lens[b] = kept;
    const int lo = min(a.first, max(n, 0)), hi = max(n - a.last, lo);  // the slots that compete
    const bool all = n <= a.budget;
    const int want = a.budget - a.first - a.last;
    const int passes = (max(n, 0) + kCluster * kSpan - 1) / (kCluster * kSpan);
    const bool choose = !all && want > 0;
    const float *mine = sh.w + threadIdx.x * (kPerThread + 1);
    auto base_of = [&](int p) { return (p * kCluster + rank) * kSpan; };
    auto stage = [&](int p) {  // a pass's weights into shared memory
        __syncthreads();
        const int base = base_of(p);
#pragma unroll 8
        for (int e = 0; e < kPerThread; ++e) {
            const int j = e * kThreads + threadIdx.x;
            sh.w[j / kPerThread * (kPerThread + 1) + j % kPerThread] =
                base + j < n ? w[base + j] : 0.0f;
        }
        __syncthreads();
    };
    uint32_t key[kPerThread];  // of the competing slots; others (and NaN) count as 0
    auto load_keys = [&](int p) {
        stage(p);
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            const int j = base_of(p) + threadIdx.x * kPerThread + e;
            key[e] = j >= lo && j < hi ? order_key(mine[e]) : 0u;
        }
    };
    uint32_t threshold = 0xFFFFFFFFu;  // keys above it are kept, and `ties` of those equal to it
    int ties = 0;
    if (choose) {
        uint32_t low = 0xFFFFFFFFu, high = 0;
        for (int p = 0; p < passes; ++p) {
            load_keys(p);
#pragma unroll
            for (int e = 0; e < kPerThread; ++e) {
                const int j = base_of(p) + threadIdx.x * kPerThread + e;
                low = min(low, j >= lo && j < hi ? key[e] : 0xFFFFFFFFu);
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
        low = __reduce_min_sync(0xFFFFFFFFu, lane < kWarps ? sh.low[lane] : 0xFFFFFFFFu);
        high = __reduce_max_sync(0xFFFFFFFFu, lane < kWarps ? sh.high[lane] : 0u);
        if (threadIdx.x == 0) {
            tell<kCluster>(sh.cta_low, low);
            tell<kCluster>(sh.cta_high, high);
        }
        meet<kCluster>();
#pragma unroll
        for (int i = 0; i < kCluster; ++i) {
            low = min(low, sh.cta_low[i]);
            high = max(high, sh.cta_high[i]);
        }
        // `need` keys are still to be taken among those that begin with `prefix`.
        const int top = low == high ? -1 : 31 - __clz(low ^ high);
        int shift = top < 0 ? -4 : top & ~3, need = want, par = 0;
        uint32_t prefix = top < 0 ? low : shift == 28 ? 0u : low >> (shift + 4) << (shift + 4);
        bool whole = false;  // all keys from the prefix on are taken
        for (; shift >= 0 && !whole; shift -= 4, par ^= 1) {
            int held = 0;  // lane d < 16: the warp's keys with digit d
            for (int p = 0; p < passes; ++p) {
                if (passes > 1)
                    load_keys(p);
                uint64_t c = 0;
#pragma unroll
                for (int e = 0; e < kPerThread; ++e) {
                    // (keys that begin otherwise add nothing)
                    const uint32_t d = (key[e] ^ prefix) >> shift;
                    c += d < 16u ? 1ull << (4 * d) : 0ull;
                }
                static_assert(kPerThread < 16, "a digit's count has four bits");
                // (two digits a word hold one pass's counts; a row of millions of slots has more
                // keys of a digit than half a word counts, so passes add up in whole ones)
                uint32_t word = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t two = (uint32_t)(c >> (8 * i));
                    const uint32_t sum =
                        __reduce_add_sync(0xFFFFFFFFu, (two & 15u) | ((two & 0xF0u) << 12));
                    word = lane >> 1 == i ? sum : word;
                }
                held += (int)((word >> (16 * (lane & 1))) & 0xFFFFu);
            }
            if (lane < 16)
                sh.digits[par][warp][lane] = held;
            __syncthreads();
            // lane d < 16 of every warp: the CTA's keys with digit d, then the cluster's
            int count = 0;
            if (kCluster == 1 || warp == 0) {
                if (lane < 16)
#pragma unroll 8
                    for (int i = 0; i < kWarps; ++i)
                        count += sh.digits[par][i][lane];
            }
            if constexpr (kCluster > 1) {
                if (warp == 0 && lane < 16)
                    for (int i = 0; i < kCluster; ++i)
                        cg::this_cluster().map_shared_rank(&sh.cta_digits[par][0][0], i)[rank * 16 + lane] =
                            count;
                meet<kCluster>();
                count = 0;
                if (lane < 16)
#pragma unroll
                    for (int i = 0; i < kCluster; ++i)
                        count += sh.cta_digits[par][i][lane];
            }
            // keys of digit d and more
            int upto = count;
#pragma unroll
            for (int m = 1; m < 16; m <<= 1) {
                const int o = __shfl_down_sync(0xFFFFFFFFu, upto, m);
                upto += lane + m < 16 ? o : 0;
            }
            const uint32_t enough = __ballot_sync(0xFFFFFFFFu, lane < 16 && upto >= need);
            const int digit = 31 - __clz(enough);
            const int at_least = __shfl_sync(0xFFFFFFFFu, upto, digit);
            const int equal = __shfl_sync(0xFFFFFFFFu, count, digit);
            need -= at_least - equal;
            prefix |= (uint32_t)digit << shift;
            whole = equal == need && prefix != 0;
        }
        threshold = whole ? prefix - 1 : prefix;
        ties = whole ? 0 : need;
    }
    int out = 0, seen = 0;
    for (int p = 0; p < passes; ++p) {
        const int from = base_of(p) + threadIdx.x * kPerThread;
        if (!choose || passes > 1)
            stage(p);
        uint32_t sure = 0, tie = 0;  // by slot of this thread
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            const int j = from + e;
            const uint32_t k = order_key(mine[e]);
            const bool competes = j >= lo && j < hi;
            if (j < n && (all || !competes || (choose && k > threshold)))
                sure |= 1u << e;
            else if (j < n && choose && k == threshold)
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
        meet<kCluster>();  // the counts of the pass before are read
        if (lane == 31) {
            sh.sure[warp] = upto_s;
            sh.ties[warp] = upto_t;
        }
        __syncthreads();
        const int s = lane < kWarps ? sh.sure[lane] : 0, t_ = lane < kWarps ? sh.ties[lane] : 0;
        int before_s = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? s : 0);
        int before_t = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? t_ : 0);
        int total_s = __reduce_add_sync(0xFFFFFFFFu, s), total_t = __reduce_add_sync(0xFFFFFFFFu, t_);
        if constexpr (kCluster > 1) {
            if (threadIdx.x == 0) {
                tell<kCluster>(sh.cta_sure, total_s);
                tell<kCluster>(sh.cta_ties, total_t);
            }
            meet<kCluster>();
            total_s = total_t = 0;
#pragma unroll
            for (int i = 0; i < kCluster; ++i) {
                before_s += i < rank ? sh.cta_sure[i] : 0;
                before_t += i < rank ? sh.cta_ties[i] : 0;
                total_s += sh.cta_sure[i];
                total_t += sh.cta_ties[i];
            }
        }
        int t = seen + before_t + upto_t - mine_t;
        int at = out + before_s + upto_s - mine_s + min(t, ties);
#pragma unroll
        for (int e = 0; e < kPerThread; ++e) {
            bool keep = (sure >> e) & 1u;
            if ((tie >> e) & 1u)
                keep = t++ < ties;
            if (keep && at < a.budget) {  // (weights that change under the call stay in bounds)
                index[at] = from + e;
                kept_w[at] = mine[e];
                ++at;
            }
        }
        out += total_s;
        seen += total_t;
    }
    for (int j = max(kept, 0) + rank * kThreads + threadIdx.x; j < a.budget;
         j += kCluster * kThreads) {
        index[j] = -1;
        kept_w[j] = 0.0f;
    }
    if constexpr (kCluster > 1)
        meet<kCluster>();  // no CTA leaves while another may still write into it
}

// Who takes a row.  One CTA where its threads hold the row in registers, 8 slots each: 256 threads
// to 2048 slots, 512 to 4096 (256 rows of 3000: 26 us; 33 with 256 threads, which read the row
// again each round; 208 with a cluster of eight, whose barriers every row pays).  Longer rows a
// cluster, of eight for a few of them (16 rows of 32000: 33 us; of two 68, of one 101), of two for
// rows of up to 8192 (16 of 8000: 23 us; eight 32, one 35) and for many (256 of 8000: 43 us; eight
// 215; 64 of 32000: 69, eight 72).
constexpr int kShortRow = 2048, kOneRow = 4096, kTwoRow = 8192, kManyRows = 64;

template <int kThreads, int kPerThread, int kCluster>
cudaError_t launch_select(const EvictArgs &a, int B, cudaStream_t s)
{
    constexpr int kBytes = sizeof(SelectShared<kThreads, kPerThread, kCluster>);
    static PerDevice ready;
    const cudaError_t e = ready.once([] {
        return cudaFuncSetAttribute(evict_select_kernel<kThreads, kPerThread, kCluster>,
                                    cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    });
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.c.heads * kCluster, B);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kBytes;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {kCluster, 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = plain_launches ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, evict_select_kernel<kThreads, kPerThread, kCluster>, a);
}

constexpr int kMoveSlots = 32;

// ---- Moving.  One CTA takes kMoveSlots kept rows of one head: keys as 16-byte pieces; values
// channel by channel.  Thread d reads the 16-byte pieces (32 slots) of channel d that hold kept
// slots, kBatch of them in flight, leaves them in a column of its own in shared memory and picks
// the nibbles, by word and shift of each slot (the same for all threads).
constexpr int kBatch = 8;

template <int D>
__global__ void __launch_bounds__(128, 8) evict_move_kernel(const __grid_constant__ EvictArgs a)
{
    __shared__ int64_t src_row[kMoveSlots];   // slot_index of the source, -1: none
    __shared__ int64_t piece_at[kMoveSlots];  // v_byte of a piece's channel 0, -1: none
    __shared__ __align__(8) uint2 place[kMoveSlots];  // a slot's word among the pieces', its shift
    __shared__ int pieces;
    __shared__ uint32_t word[4 * kBatch][D];
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
        place[lane] = make_uint2(4 * piece + ((s & 31) >> 3), 4 * (s & 7));
        if ((begins >> lane) & 1u)
            piece_at[piece] = v;
        if (lane == 0)
            pieces = __popc(begins);
    }
    __syncthreads();
    const int d = threadIdx.x;
    const bool channel = D == 128 || d < D;
    const int64_t step = (int64_t)d << (a.c.page_shift - 1);
    uint4 x[kBatch];
    auto fetch = [&](int first) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            x[i] = make_uint4(0, 0, 0, 0);
            if (channel && first + i < pieces && piece_at[first + i] >= 0)
                x[i] = *reinterpret_cast<const uint4 *>(a.c.vc + piece_at[first + i] + step);
        }
    };
    fetch(0);
    constexpr int kVecs = D / 32;  // 16-byte pieces of a row of key codes
    const int j0 = threadIdx.x / kVecs, p0 = threadIdx.x % kVecs;
    if (threadIdx.x < kMoveSlots * kVecs && src_row[j0] >= 0)
        *reinterpret_cast<uint4 *>(a.c.kc + slot_index(a.c, dpg, h, slot0 + j0) * (D / 2) +
                                   16 * p0) =
            *reinterpret_cast<const uint4 *>(a.c.kc + src_row[j0] * (D / 2) + 16 * p0);
    if (threadIdx.x < kMoveSlots && src_row[threadIdx.x] >= 0) {
        const int64_t to = slot_index(a.c, dpg, h, slot0 + threadIdx.x);
        a.c.ka[to] = a.c.ka[src_row[threadIdx.x]];
        a.c.va[to] = a.c.va[src_row[threadIdx.x]];
    }
    if (!channel)
        return;
    uint32_t out[kMoveSlots / 8] = {};
    for (int first = 0; first < pieces; first += kBatch) {
        if (first > 0)
            fetch(first);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            word[4 * i][d] = x[i].x, word[4 * i + 1][d] = x[i].y;
            word[4 * i + 2][d] = x[i].z, word[4 * i + 3][d] = x[i].w;
        }
        const uint32_t w0 = 4 * first;
        // (a slot of another batch's pieces adds nothing)
#pragma unroll
        for (int j = 0; j < kMoveSlots; ++j) {
            const uint2 f = place[j];
            const uint32_t at = f.x - w0;
            if (at < 4 * kBatch)
                out[j / 8] |= ((word[at][d] >> f.y) & 15u) << (4 * (j & 7));
        }
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
    const cudaError_t selected =
        max_len <= kShortRow ? launch_select<256, 8, 1>(a, B, s)
        : max_len <= kOneRow ? launch_select<512, 8, 1>(a, B, s)
        : max_len <= kTwoRow || (int64_t)B * a.c.heads >= kManyRows
            ? launch_select<512, 8, 2>(a, B, s)
            : launch_select<512, 8, 8>(a, B, s);
    if (selected != cudaSuccess)
        return FDLLM_ERR_CUDA;
    const dim3 grid((budget + kMoveSlots - 1) / kMoveSlots, a.c.heads, B);
    const cudaError_t e =
        a.c.D == 128 ? launch(evict_move_kernel<128>, grid, dim3(128), 0, s, true, a)
                     : launch(evict_move_kernel<64>, grid, dim3(128), 0, s, true, a);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}
