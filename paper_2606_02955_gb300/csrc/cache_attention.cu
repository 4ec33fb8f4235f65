// cache_attention.cu -- fdllm_cache_attention, and the status of the cache kernels' waits.  The
// kernels: cache_attention.cuh.
#include "cache_attention.cuh"

namespace fdllm {
namespace {

__device__ uint32_t g_status;  // sticky: a bounded wait gave up

// One warp waits on a barrier that nobody completes, as the kernels' warps wait.
__global__ void wait_probe_kernel(uint32_t *status, uint32_t tries)
{
    __shared__ __align__(8) uint64_t bar;
    if (threadIdx.x == 0) {
        mbar_init(&bar, 1);
        fence_mbar_init();
    }
    __syncthreads();
    if (!mbar_wait_at<20>(smem_addr(&bar), 0, tries))
        atomicOr(status, kDevStatTimeout);
}

}  // namespace

uint32_t *cache_status_word()
{
    static std::atomic<uint32_t *> word[kMaxCacheDevices] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxCacheDevices)
        return nullptr;
    void *p = word[dev].load(std::memory_order_relaxed);
    if (!p) {
        if (cudaGetSymbolAddress(&p, g_status) != cudaSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        word[dev].store(static_cast<uint32_t *>(p), std::memory_order_relaxed);
    }
    return static_cast<uint32_t *>(p);
}

bool check_queries(const void *q, const int64_t *strides, int dtype, int B, int Lq, int Hq,
                   int heads)
{
    return q && strides && (dtype == FDLLM_BF16 || dtype == FDLLM_FP16) && B >= 1 && Lq >= 1 &&
           Hq >= 1 && Hq <= kMaxGridYZ && Hq % heads == 0 &&
           (int64_t)Lq * (Hq / heads) < ((int64_t)1 << 30);
}

}  // namespace fdllm

using namespace fdllm;

extern "C" {

size_t fdllm_cache_attention_workspace_bytes(int B, int Lq, int Hq, int heads, int head_dim)
{
    if (B < 1 || Lq < 1 || Hq < 1 || heads < 1 || Hq % heads != 0 ||
        (head_dim != 64 && head_dim != 128))
        return 0;
    const int N = tile_rows((int64_t)Lq * (Hq / heads));
    return workspace_of(full_grid(N), N, head_dim).total;
}

fdllm_status fdllm_cache_attention(const void *q, const int64_t *q_strides, int dtype, int B,
                                   int Lq, int Hq, const fdllm_cache *cache,
                                   const int32_t *block_table, int max_pages,
                                   const int32_t *cache_lens, const void *k_new,
                                   const int64_t *k_strides, const void *v_new,
                                   const int64_t *v_strides, int Ln, const int32_t *new_lens,
                                   int causal, double scale, void *out, float *out_lse,
                                   void *workspace, size_t workspace_bytes, void *stream)
{
    return attend<false>(q, q_strides, dtype, B, Lq, Hq, cache, block_table, max_pages, cache_lens,
                         k_new, k_strides, v_new, v_strides, Ln, new_lens, causal, nullptr, scale,
                         out, out_lse, workspace, workspace_bytes, stream);
}

fdllm_status fdllm_cache_check_wait(int tries, void *stream)
{
    if (tries < 0 || tries > (int)kWaitTries)
        return FDLLM_ERR_ARG;
    uint32_t *word = cache_status_word();
    if (!word)
        return FDLLM_ERR_CUDA;
    const cudaError_t e = launch(wait_probe_kernel, dim3(1), dim3(32), 0, static_cast<cudaStream_t>(stream),
                                 false, word, tries > 0 ? (uint32_t)tries : kWaitTries);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

fdllm_status fdllm_cache_status(void *stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint32_t *word = cache_status_word(), host = 0;
    if (!word || cudaMemcpyAsync(&host, word, sizeof host, cudaMemcpyDeviceToHost, s) != cudaSuccess ||
        cudaStreamSynchronize(s) != cudaSuccess)
        return FDLLM_ERR_CUDA;
    if (host == 0)
        return FDLLM_OK;
    if (cudaMemsetAsync(word, 0, sizeof host, s) != cudaSuccess ||
        cudaStreamSynchronize(s) != cudaSuccess)
        return FDLLM_ERR_CUDA;
    return FDLLM_ERR_DEVICE;
}

}  // extern "C"
