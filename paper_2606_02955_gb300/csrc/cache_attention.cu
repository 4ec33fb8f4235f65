// cache_attention.cu -- fdllm_cache_attention and fdllm_cache_key_weights: a block's queries
// over the 4-bit prefix cache and the block's own keys.
#include <cuda_runtime.h>

#include "cache.cuh"

namespace fdllm {
namespace {

struct AttnArgs {
    CacheView c;
    const int32_t *table;     // [B, max_pages]
    int max_pages;
    const int32_t *lens;      // [B]
    const void *q;            // [B, Lq, Hq, D]
    Strides3 qs;
    int Lq, Hq, group;        // group = Hq / heads
    const void *k_new;        // [B, Ln, heads, D]
    const void *v_new;
    Strides3 ks, vs;
    int Ln;
    const int32_t *new_lens;  // [B] or null
    int causal;
    float scale;
    void *out;                // [B, Lq, Hq, D]
    float *lse;               // [B, Lq, Hq] or null
};

// A sequence's cached length, or -1 where it is out of range.
__device__ __forceinline__ int cached_len(const CacheView &c, const int32_t *lens, int max_pages,
                                          int b)
{
    const int n = lens[b];
    return n >= 0 && n <= (max_pages << c.page_shift) ? n : -1;
}

constexpr int kKeys = 128;  // keys of a step: one thread to a key

__device__ __forceinline__ float block_max(float x, float *red)
{
#pragma unroll
    for (int m = 16; m > 0; m >>= 1)
        x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, m));
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        red[threadIdx.x >> 5] = x;
    __syncthreads();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// One CTA to a query row: thread = key for the scores, thread = channel for the sum.
template <typename T, int D>
__global__ void __launch_bounds__(kKeys) attention_kernel(const __grid_constant__ AttnArgs a)
{
    __shared__ float q[D], p[kKeys], red[4];
    __shared__ int bad;
    pdl_wait();
    const int i = blockIdx.x, hq = blockIdx.y, b = blockIdx.z, h = hq / a.group;
    const T *qr = static_cast<const T *>(a.q) + b * a.qs.batch + i * a.qs.token + hq * a.qs.head;
    if (threadIdx.x < D)
        q[threadIdx.x] = to_float(qr[threadIdx.x]);
    if (threadIdx.x == 0)
        bad = 0;
    __syncthreads();
    const int n = cached_len(a.c, a.lens, a.max_pages, b);
    const int own = a.new_lens ? a.new_lens[b] : a.Ln;
    const bool wrong = n < 0 || own < 0 || own > a.Ln;
    const int seen = wrong ? 0 : (a.causal ? min(own, i + 1) : own);
    const int cached = max(n, 0);
    const int pieces = (cached + kKeys - 1) / kKeys;
    const int total = wrong ? 0 : pieces + (seen + kKeys - 1) / kKeys;
    float m = neg_inf_f(), l = 0.0f, o = 0.0f;
    const int d = threadIdx.x;
    for (int t = 0; t < total; ++t) {
        const bool in_cache = t < pieces;
        const int j0 = in_cache ? t * kKeys : (t - pieces) * kKeys;
        const int j = j0 + threadIdx.x;
        const int end = in_cache ? cached : seen;
        float s = neg_inf_f();
        if (j < end) {
            float x = 0.0f;
            if (in_cache) {
                const int pg = page_of(a.c, a.table, a.max_pages, b, j);
                if (pg < 0) {
                    bad = 1;
                } else {
                    const int64_t at = slot_index(a.c, pg, h, j);
                    const uint8_t *k = a.c.kc + at * (D / 2);
                    const uint32_t f = a.c.ka[at];
                    for (int e = 0; e < D / 2; ++e) {
                        x += q[2 * e] * fmaf(bf16_low(f), (float)(k[e] & 15), bf16_high(f));
                        x += q[2 * e + 1] * fmaf(bf16_low(f), (float)(k[e] >> 4), bf16_high(f));
                    }
                }
            } else {
                const T *k = static_cast<const T *>(a.k_new) + b * a.ks.batch + j * a.ks.token +
                             h * a.ks.head;
                for (int e = 0; e < D; ++e)
                    x += q[e] * to_float(k[e]);
            }
            s = x * a.scale;
        }
        const float top = fmaxf(m, block_max(s, red));
        const float w = j < end ? exp2f((s - top) * kLog2e) : 0.0f;
        __syncthreads();
        p[threadIdx.x] = w;
        __syncthreads();
        const float c = m == neg_inf_f() ? 0.0f : exp2f((m - top) * kLog2e);
        m = top;
        l *= c;
        o *= c;
        const int cnt = min(end - j0, kKeys);
        for (int e = 0; e < cnt; ++e) {
            l += p[e];
            if (d < D) {
                float v = 0.0f;
                if (in_cache) {
                    const int pg = page_of(a.c, a.table, a.max_pages, b, j0 + e);
                    if (pg >= 0) {
                        const uint32_t f = a.c.va[slot_index(a.c, pg, h, j0 + e)];
                        const uint32_t byte = a.c.vc[v_byte(a.c, pg, h, d, j0 + e)];
                        v = fmaf(bf16_low(f), (float)((byte >> (4 * ((j0 + e) & 1))) & 15u),
                                 bf16_high(f));
                    }
                } else {
                    v = to_float(static_cast<const T *>(a.v_new)[b * a.vs.batch +
                                                                 (j0 + e) * a.vs.token +
                                                                 h * a.vs.head + d]);
                }
                o = fmaf(p[e], v, o);
            }
        }
    }
    __syncthreads();
    const bool poison = wrong || bad != 0;
    const int64_t row = ((int64_t)b * a.Lq + i) * a.Hq + hq;
    if (d < D)
        static_cast<T *>(a.out)[row * D + d] =
            from_float<T>(poison ? nan_f() : (total ? o / l : 0.0f));
    if (d == 0 && a.lse)
        a.lse[row] = poison ? nan_f() : (total ? m + logf(l) : neg_inf_f());
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

bool check_queries(const void *q, const int64_t *strides, int dtype, int B, int Lq, int Hq,
                   int heads)
{
    return q && strides && (dtype == FDLLM_BF16 || dtype == FDLLM_FP16) && B >= 1 && Lq >= 1 &&
           Hq >= 1 && Hq <= kMaxGridYZ && Hq % heads == 0 &&
           (int64_t)Lq * (Hq / heads) < ((int64_t)1 << 30);
}

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" {

size_t fdllm_cache_attention_workspace_bytes(int B, int Lq, int Hq, int heads, int head_dim)
{
    if (B < 1 || Lq < 1 || Hq < 1 || heads < 1 || Hq % heads != 0 ||
        (head_dim != 64 && head_dim != 128))
        return 0;
    return 256;
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
    AttnArgs a = {};
    const fdllm_status st = check_cache(cache, a.c);
    if (st != FDLLM_OK)
        return st;
    if (!check_table(block_table, B, max_pages, a.c.page_shift, a.c.heads) || !cache_lens ||
        !check_queries(q, q_strides, dtype, B, Lq, Hq, a.c.heads) || Ln < 0 ||
        Ln >= (1 << 30) || (Ln > 0 && (!k_new || !v_new || !k_strides || !v_strides)) ||
        (causal != 0 && causal != 1) || !std::isfinite(scale) || !out)
        return FDLLM_ERR_ARG;
    const int64_t none[1] = {0};
    if (!aligned16(q, q_strides, 3, 2) || !aligned16(out, none, 0, 2) ||
        (Ln > 0 && (!aligned16(k_new, k_strides, 3, 2) || !aligned16(v_new, v_strides, 3, 2))))
        return FDLLM_ERR_ALIGN;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
        workspace_bytes <
            fdllm_cache_attention_workspace_bytes(B, Lq, Hq, a.c.heads, a.c.D))
        return FDLLM_ERR_WORKSPACE;
    a.table = block_table;
    a.max_pages = max_pages;
    a.lens = cache_lens;
    a.q = q;
    a.qs = strides3(q_strides);
    a.Lq = Lq;
    a.Hq = Hq;
    a.group = Hq / a.c.heads;
    if (Ln > 0) {
        a.k_new = k_new;
        a.v_new = v_new;
        a.ks = strides3(k_strides);
        a.vs = strides3(v_strides);
    }
    a.Ln = Ln;
    a.new_lens = new_lens;
    a.causal = causal;
    a.scale = (float)scale;
    a.out = out;
    a.lse = out_lse;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid(Lq, Hq, B);
    const bool bf = dtype == FDLLM_BF16, wide = a.c.D == 128;
    const cudaError_t e =
        bf ? (wide ? launch(attention_kernel<__nv_bfloat16, 128>, grid, dim3(kKeys), 0, s, true, a)
                   : launch(attention_kernel<__nv_bfloat16, 64>, grid, dim3(kKeys), 0, s, true, a))
           : (wide ? launch(attention_kernel<__half, 128>, grid, dim3(kKeys), 0, s, true, a)
                   : launch(attention_kernel<__half, 64>, grid, dim3(kKeys), 0, s, true, a));
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

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
