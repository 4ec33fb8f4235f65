// cache_tree.cu -- fdllm_tree_mask and fdllm_cache_tree_attention: a tree of drafted tokens over the
// 4-bit prefix cache.  A node's query sees the cached keys and the keys of its ancestors and itself;
// the attention's kernels are those of cache_attention.cuh with a bit for each pair of nodes.
#include "cache_attention.cuh"

namespace fdllm {
namespace {

constexpr int kMaxNodes = FDLLM_MAX_L;

struct MaskArgs {
    const int32_t *parents;  // [B, M]
    const int32_t *lens;     // [B] or null
    int M, words;
    uint32_t *mask;          // [B, M, words]
    int32_t *depth;          // [B, M] or null
};

// One CTA a sequence, a thread to a word of a node's row of bits.  Each turn a node's row takes in the
// row of the node that its walk up has reached, and the walk doubles its length: as many turns as
// the depth has bits.  Bound by the turns' latencies: 32
// trees of 48 nodes 2 to 3 us, two of 255 3 to 5 (a warp to a row 8 to 15), by the depth.
__global__ void __launch_bounds__(1024) tree_mask_kernel(const __grid_constant__ MaskArgs a)
{
    extern __shared__ uint32_t rows[];  // [M][words]
    __shared__ short up[2][kMaxNodes], dist[2][kMaxNodes];
    pdl_wait();
    const int b = blockIdx.x;
    const int log = 32 - __clz(a.words - 1), all = 1 << log;  // words of a row, those not there too
    const int n = a.lens ? min(max(a.lens[b], 0), a.M) : a.M;
    for (int i = threadIdx.x; i < a.M; i += blockDim.x) {
        const int p = i > 0 && i < n ? a.parents[(int64_t)b * a.M + i] : -1;
        const bool hung = p >= 0 && p < i;
        up[0][i] = hung ? p : -1;
        dist[0][i] = hung ? 1 : 0;
    }
    for (int x = threadIdx.x; x < a.M << log; x += blockDim.x) {
        const int i = x >> log, w = x & (all - 1);
        if (w < a.words)
            rows[i * a.words + w] = i < n && (i >> 5) == w ? 1u << (i & 31) : 0u;
    }
    int from = 0, more = 1;
    while (more) {
        __syncthreads();
        // (a row may be read while it takes bits in: they are ancestors' all the same)
        for (int x = threadIdx.x; x < n << log; x += blockDim.x) {
            const int i = x >> log, w = x & (all - 1), p = up[from][i];
            if (p >= 0 && w < a.words)
                rows[i * a.words + w] |= *(volatile uint32_t *)&rows[p * a.words + w];
        }
        int on = 0;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int p = up[from][i], q = p >= 0 ? up[from][p] : -1;
            up[from ^ 1][i] = q;
            dist[from ^ 1][i] = dist[from][i] + (p >= 0 ? dist[from][p] : 0);
            on |= q >= 0;
        }
        from ^= 1;
        more = __syncthreads_or(on);
    }
    __syncthreads();
    for (int x = threadIdx.x; x < a.M * a.words; x += blockDim.x)
        a.mask[(int64_t)b * a.M * a.words + x] = rows[x];
    if (a.depth)
        for (int i = threadIdx.x; i < a.M; i += blockDim.x)
            a.depth[(int64_t)b * a.M + i] = i < n ? dist[from][i] : -1;
}

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_tree_mask(const int32_t *parents, const int32_t *lens, int B, int M,
                             uint32_t *out_mask, int32_t *out_depth, void *stream)
{
    if (!parents || !out_mask || B < 1 || B > kMaxGridYZ || M < 1 || M > kMaxNodes)
        return FDLLM_ERR_ARG;
    MaskArgs a = {parents, lens, M, (M + 31) / 32, out_mask, out_depth};
    static PerDevice ready;
    if (ready.once([] {
            return cudaFuncSetAttribute(tree_mask_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                        kMaxNodes * (kMaxNodes / 32) * 4);
        }) != cudaSuccess)
        return FDLLM_ERR_CUDA;
    const int threads = M <= 32 ? 128 : M <= 128 ? 512 : 1024;
    const cudaError_t e = launch(tree_mask_kernel, dim3(B), dim3(threads), (size_t)M * a.words * 4,
                                 static_cast<cudaStream_t>(stream), true, a);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

fdllm_status fdllm_cache_tree_attention(const void *q, const int64_t *q_strides, int dtype, int B,
                                        int Lq, int Hq, const fdllm_cache *cache,
                                        const int32_t *block_table, int max_pages,
                                        const int32_t *cache_lens, const void *k_new,
                                        const int64_t *k_strides, const void *v_new,
                                        const int64_t *v_strides, int Ln, const int32_t *new_lens,
                                        const uint32_t *mask, double scale, void *out,
                                        float *out_lse, void *workspace, size_t workspace_bytes,
                                        void *stream)
{
    return attend<true>(q, q_strides, dtype, B, Lq, Hq, cache, block_table, max_pages, cache_lens,
                        k_new, k_strides, v_new, v_strides, Ln, new_lens, 0, mask, scale, out,
                        out_lse, workspace, workspace_bytes, stream);
}

}  // extern "C"
