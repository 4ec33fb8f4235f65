// vocab_rows.cuh -- what the kernels that walk rows of logits share (distill.cu, verify.cu): rows of
// any length and alignment as 16-byte vectors with loose ends, sums of exponentials with a running
// maximum, and reductions over a CTA in a fixed order.
#pragma once

#include <cfloat>
#include <cstdint>

#include "cache.cuh"

namespace fdllm {

constexpr int kMaxRowV = 1 << 20;  // vocabulary of these operators: a bit for each token fits a CTA

inline bool rows_dtype(int d) { return d == FDLLM_BF16 || d == FDLLM_FP16 || d == FDLLM_FP32; }
inline int rows_esize(int d) { return d == FDLLM_FP32 ? 4 : 2; }

#ifdef __CUDACC__

// A row of V values: `head` of them before the first 16-byte boundary, `vecs` whole vectors, and
// the rest.
template <typename T>
struct RowSpan {
    static constexpr int E = 16 / sizeof(T);
    const T *row;
    int V, head, vecs;
    __device__ __forceinline__ RowSpan(const T *p, int n) : row(p), V(n)
    {
        head = min(n, (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(p)) & 15u) / (int)sizeof(T));
        vecs = (n - head) / E;
    }
    __device__ __forceinline__ const uint4 *vectors() const
    {
        return reinterpret_cast<const uint4 *>(row + head);
    }
    __device__ __forceinline__ int tail() const { return head + vecs * E; }  // first value behind
};

// The values of a 16-byte vector.
template <typename T>
__device__ __forceinline__ void widen(const uint4 &r, float (&x)[16 / sizeof(T)])
{
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else if constexpr (__is_same(T, __nv_bfloat16)) {
            x[2 * i] = bf16_low(w[i]);
            x[2 * i + 1] = bf16_high(w[i]);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}

template <typename T>
__device__ __forceinline__ uint4 narrow(const float (&x)[16 / sizeof(T)])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4)
            w[i] = __float_as_uint(x[i]);
        else
            w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Sum of 2^((x - m) c) with the running maximum m.  A NaN or a +inf makes z NaN; before the first
// finite value, and where all are -inf, m is -FLT_MAX and z is 0.  The difference is taken before
// the product, so values of any size keep what tells them apart.
struct ExpSum {
    float m = -FLT_MAX, z = 0.0f;

    __device__ __forceinline__ void raise(float to, float c)
    {
        if (to > m) {
            z *= ex2_mufu((m - to) * c);
            m = to;
        }
    }
    __device__ __forceinline__ void add(float x, float c)
    {
        raise(x, c);
        z += ex2_mufu((x - m) * c);
    }
    __device__ __forceinline__ void merge(const ExpSum &o, float c)
    {
        const float top = fmaxf(m, o.m);
        z = z * ex2_mufu((m - top) * c) + o.z * ex2_mufu((o.m - top) * c);
        m = top;
    }
};

__device__ __forceinline__ ExpSum warp_sum(ExpSum s, float c)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        ExpSum t;
        t.m = __shfl_xor_sync(0xFFFFFFFFu, s.m, o);
        t.z = __shfl_xor_sync(0xFFFFFFFFu, s.z, o);
        s.merge(t, c);
    }
    return s;
}

// The warp's largest value (no NaN among them).
__device__ __forceinline__ float warp_most(float x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}

__device__ __forceinline__ bool finite_f(float x) { return fabsf(x) <= FLT_MAX; }

#endif  // __CUDACC__

}  // namespace fdllm
