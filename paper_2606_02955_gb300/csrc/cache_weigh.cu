// cache_weigh.cu -- fdllm_cache_key_weights: the attention that each cached key receives.
#include <cuda_runtime.h>

#include "cache.cuh"

namespace fdllm {
namespace {

constexpr int kKeys = 128;

__device__ __forceinline__ int cached_len(const CacheView &c, const int32_t *lens, int max_pages,
                                          int b)
{
    const int n = lens[b];
    return n >= 0 && n <= (max_pages << c.page_shift) ? n : -1;
}

struct WeighArgs {
    CacheView c;
    const int32_t *table;
    int max_pages;
    const int32_t *lens;
    const void *q;
    Strides3 qs;
    int Lq, Hq, group;
    const float *lse;         // [B, Lq, Hq]
    float scale;
    const float *in;          // [B, heads, max_len] or null
    float *out;
    int max_len;
};

// One thread to a key.
template <typename T, int D>
__global__ void __launch_bounds__(kKeys) weigh_kernel(const __grid_constant__ WeighArgs a)
{
    __shared__ float q[D];
    pdl_wait();
    const int j = blockIdx.x * kKeys + threadIdx.x, h = blockIdx.y, b = blockIdx.z;
    int n = cached_len(a.c, a.lens, a.max_pages, b);
    if (n > a.max_len)
        n = -1;
    const int pg = j < n ? page_of(a.c, a.table, a.max_pages, b, j) : -1;
    float k[D];
    if (pg >= 0) {
        const int64_t at = slot_index(a.c, pg, h, j);
        const uint32_t f = a.c.ka[at];
        for (int e = 0; e < D / 2; ++e) {
            const uint32_t w = a.c.kc[at * (D / 2) + e];
            k[2 * e] = fmaf(bf16_low(f), (float)(w & 15), bf16_high(f));
            k[2 * e + 1] = fmaf(bf16_low(f), (float)(w >> 4), bf16_high(f));
        }
    }
    float sum = 0.0f;
    for (int r = 0; r < a.Lq * a.group; ++r) {
        const int i = r / a.group, hq = h * a.group + r % a.group;
        __syncthreads();
        if (threadIdx.x < D)
            q[threadIdx.x] = to_float(static_cast<const T *>(
                a.q)[b * a.qs.batch + i * a.qs.token + hq * a.qs.head + threadIdx.x]);
        __syncthreads();
        const float lse = a.lse[((int64_t)b * a.Lq + i) * a.Hq + hq];
        if (pg >= 0 && lse != neg_inf_f()) {
            float x = 0.0f;
#pragma unroll
            for (int e = 0; e < D; ++e)
                x += q[e] * k[e];
            sum += exp2f((x * a.scale - lse) * kLog2e);
        }
    }
    if (j < a.max_len) {
        const int64_t at = ((int64_t)b * a.c.heads + h) * a.max_len + j;
        float y = 0.0f;
        if (n < 0 || (j < n && pg < 0))
            y = nan_f();
        else if (j < n)
            y = (a.in ? a.in[at] : 0.0f) + sum;
        a.out[at] = y;
    }
}

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_cache_key_weights(const void *q, const int64_t *q_strides, int dtype, int B,
                                     int Lq, int Hq, const fdllm_cache *cache,
                                     const int32_t *block_table, int max_pages,
                                     const int32_t *cache_lens, const float *lse, double scale,
                                     const float *weights_in, float *weights_out, int max_len,
                                     void *stream)
{
    WeighArgs a = {};
    const fdllm_status st = check_cache(cache, a.c);
    if (st != FDLLM_OK)
        return st;
    if (!check_table(block_table, B, max_pages, a.c.page_shift, a.c.heads) || !cache_lens ||
        !check_queries(q, q_strides, dtype, B, Lq, Hq, a.c.heads) || !lse ||
        !std::isfinite(scale) || !weights_out || max_len < 1 || max_len >= (1 << 30))
        return FDLLM_ERR_ARG;
    if (!aligned16(q, q_strides, 3, 2))
        return FDLLM_ERR_ALIGN;
    a.table = block_table;
    a.max_pages = max_pages;
    a.lens = cache_lens;
    a.q = q;
    a.qs = strides3(q_strides);
    a.Lq = Lq;
    a.Hq = Hq;
    a.group = Hq / a.c.heads;
    a.lse = lse;
    a.scale = (float)scale;
    a.in = weights_in;
    a.out = weights_out;
    a.max_len = max_len;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid((max_len + kKeys - 1) / kKeys, a.c.heads, B);
    const bool bf = dtype == FDLLM_BF16, wide = a.c.D == 128;
    const cudaError_t e =
        bf ? (wide ? launch(weigh_kernel<__nv_bfloat16, 128>, grid, dim3(kKeys), 0, s, true, a)
                   : launch(weigh_kernel<__nv_bfloat16, 64>, grid, dim3(kKeys), 0, s, true, a))
           : (wide ? launch(weigh_kernel<__half, 128>, grid, dim3(kKeys), 0, s, true, a)
                   : launch(weigh_kernel<__half, 64>, grid, dim3(kKeys), 0, s, true, a));
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

}  // extern "C"
