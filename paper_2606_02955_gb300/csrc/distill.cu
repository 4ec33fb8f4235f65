// distill.cu -- fdllm_distill_loss, fdllm_distill_grad and fdllm_distill_step: the loss that trains a
// model on its teacher's top logits at the masked positions, and its gradient.
//
// Mathematics.  A row x of logits, temperature T, q = softmax(x / T); the teacher's probabilities p_k
// of its listed tokens, their sum P, and (where the teacher's log-sum-exp is given) the rest R of
// the teacher's mass, against the rest r = sum q_v over the tokens that are not listed:
//   loss = sum_k p_k (log p_k - log q_k) + R (log R - log r)
//   d loss / d x_v = (q_v (P + R) - p_v) / T                       for a listed token,
//                    s_v (r (P + R) - R) / T,  s_v = q_v / r       for another.
// The tokens that are not listed are summed by themselves, relative to their own maximum: log r
// and s_v keep their accuracy where the listed tokens hold all of the student's mass but e^-100,
// and r is never a difference of near numbers.  Listed tokens are marked by a bit each in shared
// memory and left out of the sum as the row goes by.
#include <cuda_runtime.h>

#include "vocab_rows.cuh"

namespace fdllm {
namespace {

constexpr int kMaxTop = 1024;
constexpr int kThreads = 512;

struct DistillArgs {
    const void *logits;      // [rows, V]
    int64_t rows;
    int V;
    const uint8_t *mask;     // [rows]
    const int32_t *index;    // [rows, K]
    const void *top;         // [rows, K]
    int top_dtype;
    int K;
    const float *lse;        // [rows] or null
    float inv_t;             // 1 / temperature
    float temperature;
    const float *grad_loss;  // [rows]
    float *loss;             // [rows]
    float4 *stats_out;       // [rows]: what the gradient needs of a row
    const float4 *stats_in;
    void *grad;              // [rows, V]
};

__device__ __forceinline__ float top_value(const DistillArgs &a, int64_t i)
{
    if (a.top_dtype == FDLLM_FP32)
        return static_cast<const float *>(a.top)[i];
    if (a.top_dtype == FDLLM_BF16)
        return __bfloat162float(static_cast<const __nv_bfloat16 *>(a.top)[i]);
    return __half2float(static_cast<const __half *>(a.top)[i]);
}

// Sum (or maximum) over the CTA, the same bits in every thread.
template <typename F>
__device__ __forceinline__ float cta_reduce(float x, float *warps, F f)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        x = f(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        warps[threadIdx.x >> 5] = x;
    __syncthreads();
    x = warps[0];
    for (int i = 1; i < kThreads / 32; ++i)
        x = f(x, warps[i]);
    return x;
}

struct Add {
    __device__ float operator()(float a, float b) const { return a + b; }
};
struct Most {  // a NaN stays
    __device__ float operator()(float a, float b) const
    {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
        return r;
    }
};

// kSum: the row's sums are taken (else they are given); kGrad: the gradient is written.
template <typename T, bool kSum, bool kGrad>
__global__ void __launch_bounds__(kThreads) distill_kernel(const __grid_constant__ DistillArgs a)
{
    constexpr int E = 16 / sizeof(T);
    constexpr int kMine = kMaxTop / kThreads;  // listed tokens of a thread
    extern __shared__ __align__(16) uint32_t listed[];  // a bit for each token
    __shared__ int idx[kMaxTop];
    __shared__ float p[kMaxTop];
    __shared__ float warps[kThreads / 32];
    __shared__ ExpSum sums[kThreads / 32];
    __shared__ int twice;
    pdl_wait();
    const int tid = threadIdx.x;
    const float c = a.inv_t * kLog2e;
    for (int i = tid; i < (a.V + 31) / 32; i += kThreads)
        listed[i] = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        T *grad = static_cast<T *>(a.grad) + row * a.V;
        if (!a.mask[row]) {
            if (kGrad) {
                const RowSpan<T> g(grad, a.V);
                for (int i = tid; i < g.head; i += kThreads)
                    grad[i] = from_float<T>(0.0f);
                for (int i = tid; i < g.vecs; i += kThreads)
                    reinterpret_cast<uint4 *>(grad + g.head)[i] = make_uint4(0, 0, 0, 0);
                for (int i = g.tail() + tid; i < a.V; i += kThreads)
                    grad[i] = from_float<T>(0.0f);
            }
            if (kSum && tid == 0) {
                a.loss[row] = 0.0f;
                if (a.stats_out)
                    a.stats_out[row] = make_float4(0, 0, 0, 0);
            }
            continue;
        }
        const RowSpan<T> s(static_cast<const T *>(a.logits) + row * a.V, a.V);
        // ---- the teacher's probabilities, and the student's logits of its tokens
        int v[kMine];
        float m[kMine], x[kMine];
        if (tid == 0)
            twice = 0;
        __syncthreads();
        float most = -FLT_MAX;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            const int k = tid + j * kThreads;
            v[j] = -1;
            m[j] = x[j] = neg_inf_f();
            if (k < a.K) {
                const int at = a.index[row * a.K + k];
                if (at >= 0 && at < a.V) {
                    v[j] = at;
                    m[j] = __fdiv_rn(top_value(a, row * a.K + k), a.temperature);
                    x[j] = to_float(s.row[at]);
                    if ((atomicOr(&listed[at >> 5], 1u << (at & 31)) >> (at & 31)) & 1u)
                        twice = 1;
                }
                idx[k] = v[j];
                most = Most()(most, m[j]);
            }
        }
        most = a.lse ? a.lse[row] : cta_reduce(most, warps, Most());
        float P = 0.0f, R = 0.0f;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            m[j] = v[j] >= 0 ? expf(m[j] - most) : 0.0f;
            P += m[j];
        }
        P = cta_reduce(P, warps, Add());
        if (a.lse) {
            R = fmaxf(1.0f - P, 0.0f);
        } else if (P != 0.0f) {
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                m[j] = __fdiv_rn(m[j], P);
            P = P == P ? 1.0f : P;
        }
        __syncthreads();
        if (twice) {  // a token listed more than once: its masses count together, in its first place
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (tid + j * kThreads < a.K)
                    p[tid + j * kThreads] = m[j];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                const int k = tid + j * kThreads;
                if (v[j] < 0)
                    continue;
                m[j] = 0.0f;
                for (int i = 0; i < a.K; ++i)
                    if (idx[i] == v[j]) {
                        if (i < k) {
                            v[j] = -1;
                            x[j] = neg_inf_f();
                            break;
                        }
                        m[j] += p[i];
                    }
            }
        }
        float M, Z, r;
        ExpSum rest;
        if (kSum) {
            // ---- the tokens that are not listed
            auto value = [&](int i) {
                return (listed[i >> 5] >> (i & 31)) & 1u ? neg_inf_f() : to_float(s.row[i]);
            };
            for (int i = tid; i < s.head; i += kThreads)
                rest.add(value(i), c);
            for (int i = s.tail() + tid; i < a.V; i += kThreads)
                rest.add(value(i), c);
            for (int i = tid; i < s.vecs; i += kThreads) {
                float y[E];
                widen<T>(s.vectors()[i], y);
                const int at = s.head + i * E;
                float top = -FLT_MAX;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    y[e] = (listed[(at + e) >> 5] >> ((at + e) & 31)) & 1u ? neg_inf_f() : y[e];
                    top = fmaxf(top, y[e]);
                }
                rest.raise(top, c);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    rest.z += ex2_mufu((y[e] - rest.m) * c);
            }
            rest = warp_sum(rest, c);
            __syncthreads();
            if ((tid & 31) == 0)
                sums[tid >> 5] = rest;
            __syncthreads();
            rest = sums[0];
            for (int i = 1; i < kThreads / 32; ++i)
                rest.merge(sums[i], c);
            // ---- all tokens: the listed ones among them
            M = rest.m;
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                M = fmaxf(M, x[j]);
            M = cta_reduce(M, warps, Most());
            Z = 0.0f;
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (v[j] >= 0)
                    Z += ex2_mufu((x[j] - M) * c);
            Z = cta_reduce(Z, warps, Add());
            Z += rest.z * ex2_mufu((rest.m - M) * c);
            if (!(Z > 0.0f && Z <= FLT_MAX) || !finite_f(M))
                Z = nan_f();
            const float log_z = logf(Z);
            float loss = 0.0f;
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (v[j] >= 0 && m[j] != 0.0f)
                    loss += m[j] * (logf(m[j]) - ((x[j] - M) * a.inv_t - log_z));
            loss = cta_reduce(loss, warps, Add());
            if (rest.z == 0.0f)
                R = 0.0f;
            if (R > 0.0f)
                loss += R * (logf(R) - ((rest.m - M) * a.inv_t + logf(rest.z) - log_z));
            if (Z != Z)
                loss = Z;
            if (tid == 0) {
                a.loss[row] = loss;
                if (a.stats_out)
                    a.stats_out[row] = make_float4(M, Z, rest.m, rest.z);
            }
        } else {
            const float4 st = a.stats_in[row];
            M = st.x;
            Z = st.y;
            rest.m = st.z;
            rest.z = st.w;
            if (rest.z == 0.0f)
                R = 0.0f;
        }
        if (kGrad) {
            const float scale = a.grad_loss[row] * a.inv_t;
            r = rest.z * ex2_mufu((rest.m - M) * c) / Z;
            // of s_v relative to the rest's maximum
            const float f = rest.z == 0.0f ? (Z == Z ? 0.0f : Z)
                                           : scale * (r * (P + R) - R) / rest.z;
            auto of = [&](float y) { return ex2_mufu((y - rest.m) * c) * f; };
            for (int i = tid; i < s.head; i += kThreads)
                grad[i] = from_float<T>(of(to_float(s.row[i])));
            for (int i = s.tail() + tid; i < a.V; i += kThreads)
                grad[i] = from_float<T>(of(to_float(s.row[i])));
            for (int i = tid; i < s.vecs; i += kThreads) {
                float y[E];
                widen<T>(s.vectors()[i], y);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    y[e] = of(y[e]);
                reinterpret_cast<uint4 *>(grad + s.head)[i] = narrow<T>(y);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (v[j] >= 0)
                    grad[v[j]] = from_float<T>(
                        scale * (ex2_mufu((x[j] - M) * c) / Z * (P + R) - m[j]));
        }
        __syncthreads();
        for (int k = tid; k < a.K; k += kThreads)
            if (idx[k] >= 0)
                listed[idx[k] >> 5] = 0;
    }
}

template <typename T>
cudaError_t launch_distill(const DistillArgs &a, bool sum, bool grad, cudaStream_t s)
{
    const size_t smem = (size_t)((a.V + 31) / 32) * 4;
    static PerDevice ready;
    cudaError_t e = ready.once([] {
        const int most = kMaxRowV / 8;
        cudaError_t r = cudaFuncSetAttribute(distill_kernel<T, true, false>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (r == cudaSuccess)
            r = cudaFuncSetAttribute(distill_kernel<T, true, true>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (r == cudaSuccess)
            r = cudaFuncSetAttribute(distill_kernel<T, false, true>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        return r;
    });
    if (e != cudaSuccess)
        return e;
    const int64_t most = (int64_t)sm_count() * 2;
    const dim3 grid((unsigned)(a.rows < most ? a.rows : most)), block(kThreads);
    if (sum && grad)
        return launch(distill_kernel<T, true, true>, grid, block, smem, s, true, a);
    if (sum)
        return launch(distill_kernel<T, true, false>, grid, block, smem, s, true, a);
    return launch(distill_kernel<T, false, true>, grid, block, smem, s, true, a);
}

// What the three entry points check alike.
fdllm_status check_distill(DistillArgs &a, const void *logits, int dtype, int B, int L, int V,
                           const uint8_t *mask, const int32_t *top_index, const void *top_logits,
                           int top_dtype, int K, const float *teacher_lse, double temperature)
{
    if (!rows_dtype(dtype) || !rows_dtype(top_dtype) || B < 1 || L < 1 ||
        (int64_t)B * L >= ((int64_t)1 << 31) || V < 1 || V > kMaxRowV || K < 1 || K > kMaxTop ||
        !logits || !mask || !top_index || !top_logits || !std::isfinite(temperature) ||
        !(temperature >= 1e-6 && temperature <= 1e6))
        return FDLLM_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(logits) & 15u) != 0)
        return FDLLM_ERR_ALIGN;
    a.logits = logits;
    a.rows = (int64_t)B * L;
    a.V = V;
    a.mask = mask;
    a.index = top_index;
    a.top = top_logits;
    a.top_dtype = top_dtype;
    a.K = K;
    a.lse = teacher_lse;
    a.temperature = (float)temperature;
    a.inv_t = (float)(1.0 / temperature);
    return FDLLM_OK;
}

fdllm_status run_distill(const DistillArgs &a, int dtype, bool sum, bool grad, void *stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == FDLLM_BF16   ? launch_distill<__nv_bfloat16>(a, sum, grad, s)
                          : dtype == FDLLM_FP16 ? launch_distill<__half>(a, sum, grad, s)
                                                : launch_distill<float>(a, sum, grad, s);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_distill_loss(const void *logits, int dtype, int B, int L, int V,
                                const uint8_t *mask, const int32_t *top_index,
                                const void *top_logits, int top_dtype, int K,
                                const float *teacher_lse, double temperature, float *out_loss,
                                float *out_stats, void *stream)
{
    DistillArgs a = {};
    const fdllm_status st = check_distill(a, logits, dtype, B, L, V, mask, top_index, top_logits,
                                          top_dtype, K, teacher_lse, temperature);
    if (st != FDLLM_OK)
        return st;
    if (!out_loss)
        return FDLLM_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(out_stats) & 15u) != 0)
        return FDLLM_ERR_ALIGN;
    a.loss = out_loss;
    a.stats_out = reinterpret_cast<float4 *>(out_stats);
    return run_distill(a, dtype, true, false, stream);
}

fdllm_status fdllm_distill_grad(const void *logits, int dtype, int B, int L, int V,
                                const uint8_t *mask, const int32_t *top_index,
                                const void *top_logits, int top_dtype, int K,
                                const float *teacher_lse, double temperature, const float *stats,
                                const float *grad_loss, void *out_grad, void *stream)
{
    DistillArgs a = {};
    const fdllm_status st = check_distill(a, logits, dtype, B, L, V, mask, top_index, top_logits,
                                          top_dtype, K, teacher_lse, temperature);
    if (st != FDLLM_OK)
        return st;
    if (!stats || !grad_loss || !out_grad)
        return FDLLM_ERR_ARG;
    if (((reinterpret_cast<uintptr_t>(stats) | reinterpret_cast<uintptr_t>(out_grad)) & 15u) != 0)
        return FDLLM_ERR_ALIGN;
    a.stats_in = reinterpret_cast<const float4 *>(stats);
    a.grad_loss = grad_loss;
    a.grad = out_grad;
    return run_distill(a, dtype, false, true, stream);
}

fdllm_status fdllm_distill_step(const void *logits, int dtype, int B, int L, int V,
                                const uint8_t *mask, const int32_t *top_index,
                                const void *top_logits, int top_dtype, int K,
                                const float *teacher_lse, double temperature,
                                const float *grad_loss, float *out_loss, void *out_grad,
                                void *stream)
{
    DistillArgs a = {};
    const fdllm_status st = check_distill(a, logits, dtype, B, L, V, mask, top_index, top_logits,
                                          top_dtype, K, teacher_lse, temperature);
    if (st != FDLLM_OK)
        return st;
    if (!grad_loss || !out_loss || !out_grad)
        return FDLLM_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(out_grad) & 15u) != 0)
        return FDLLM_ERR_ALIGN;
    a.grad_loss = grad_loss;
    a.loss = out_loss;
    a.grad = out_grad;
    return run_distill(a, dtype, true, true, stream);
}

}  // extern "C"
