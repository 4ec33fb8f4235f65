// vocab_rows.cuh -- what the kernels that walk rows of logits share (distill.cu, verify.cu): rows of
// any length and alignment as 16-byte vectors with loose ends, sums of exponentials with a running
// maximum, and reductions over a CTA in a fixed order.
#pragma once

#include <cfloat>
#include <cstdint>
#include <type_traits>

#include "cache.cuh"
#include "cache_tc.cuh"
#include "ptx.cuh"

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

// The largest of a vector's values; NaN where one is.
template <typename T>
__device__ __forceinline__ float vector_most(const uint4 &r)
{
    if constexpr (sizeof(T) == 4) {
        return fmax_nan(fmax_nan(__uint_as_float(r.x), __uint_as_float(r.y)),
                        fmax_nan(__uint_as_float(r.z), __uint_as_float(r.w)));
    } else {
        using P = std::conditional_t<__is_same(T, __nv_bfloat16), __nv_bfloat162, __half2>;
        auto as = [](const uint32_t &w) { return *reinterpret_cast<const P *>(&w); };
        const P m = __hmax2_nan(__hmax2_nan(as(r.x), as(r.y)), __hmax2_nan(as(r.z), as(r.w)));
        return fmax_nan(to_float(m.x), to_float(m.y));
    }
}

template <typename T>
__device__ __forceinline__ constexpr uint32_t no_values()  // a word of -inf
{
    return sizeof(T) == 4 ? 0xFF800000u : __is_same(T, __nv_bfloat16) ? 0xFF80FF80u : 0xFC00FC00u;
}

// A thread's sum of 2^((x - m) c) over its vectors.  m is a reference, not the maximum: it moves only
// where a value exceeds it by kSlack, so that few vectors pay for that, and terms stay below 2^kSlack.
// Below kFar the terms are 2^(x c - r), r = m c rounded, in one operation: the product is exact
// there, and what r's rounding leaves, at most 2^-3 and the same for all terms, is taken out at the
// end.  Beyond kFar, x less m comes first.
constexpr float kSlack = 12.0f, kFar = 2097152.0f;

struct Summed {
    ExpSum z;
    float r = 0.0f;
    bool far = true;  // (so that a first value of -FLT_MAX, which moves nothing, counts 1)

    template <typename T, int N>
    __device__ __forceinline__ void add(const uint4 (&x)[N], float c)
    {
        constexpr int E = 16 / sizeof(T);
        float top = vector_most<T>(x[0]);
#pragma unroll
        for (int n = 1; n < N; ++n)
            top = fmax_nan(top, vector_most<T>(x[n]));
        // (a NaN fails the test as well, and moves nothing: its term makes the sum NaN)
        if (!((top - z.m) * c <= kSlack)) {
            if (top > z.m) {
                settle(c);
                z.raise(top, c);
                r = z.m * c;
                far = !(fabsf(r) < kFar);
                if (!far)
                    z.z *= ex2_mufu(fmaf(z.m, c, -r));
            }
        }
        uint64_t s2 = 0;
        auto terms = [&](auto far_tag) {
            constexpr bool kIsFar = decltype(far_tag)::value;
            const uint64_t c2 = f2(c, c), n2 = kIsFar ? f2(-z.m, -z.m) : f2(-r, -r);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float y[E];
                widen<T>(x[n], y);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    float t0, t1;
                    const uint64_t y2 = f2(y[e], y[e + 1]);
                    un2(kIsFar ? mul2(add2(y2, n2), c2) : fma2(y2, c2, n2), t0, t1);
                    s2 = add2(s2, f2(ex2_mufu(t0), ex2_mufu(t1)));
                }
            }
        };
        if (__builtin_expect(far, 0))
            terms(std::true_type{});
        else
            terms(std::false_type{});
        float s0, s1;
        un2(s2, s0, s1);
        z.z += s0 + s1;
    }
    // The sum relative to m itself.
    __device__ __forceinline__ void settle(float c)
    {
        if (!far && z.z != 0.0f)
            z.z *= ex2_mufu(-fmaf(z.m, c, -r));
        far = true;
    }
};

// The cluster's barrier, in its two halves.  A CTA may leave behind its last arrival.
__device__ __forceinline__ void cluster_arrive_relaxed()  // (orders no memory)
{
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive()
{
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ bool finite_f(float x) { return fabsf(x) <= FLT_MAX; }

// Clusters of `ranks` CTAs, one to an SM, that the GPU holds at once.
template <typename K>
int clusters_held(K kern, int threads, int smem, int ranks)
{
    if (ranks == 1)
        return sm_count();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(sm_count() / ranks * ranks));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)ranks, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = sm_count() / ranks;
    }
    return n;
}

#endif  // __CUDACC__

}  // namespace fdllm
