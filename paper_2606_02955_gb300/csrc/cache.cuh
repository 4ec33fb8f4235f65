// cache.cuh -- what the kernels of the 4-bit prefix cache share: the view of a cache, page
// lookup, conversion of rows of 16-bit or 32-bit values, argument checks and launches.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>

#include "fdllm.h"
#include "fdllm_internal.cuh"

namespace fdllm {

// fdllm_cache as the kernels see it.
struct CacheView {
    uint8_t *kc;       // [pages, heads, page, D/2]
    uint8_t *vc;       // [pages, heads, D, page/2]
    uint32_t *ka;      // [pages, heads, page]: scale in the low half, offset in the high
    uint32_t *va;
    int pages;
    int heads;
    int page_shift;    // log2 of the page size
    int D;
};

struct Strides3 {
    int64_t batch, token, head;
};

// A cache's sizes and pointers, checked on the host.
inline fdllm_status check_cache(const fdllm_cache *c, CacheView &v)
{
    if (!c || !c->k_codes || !c->v_codes || !c->k_affine || !c->v_affine || c->pages < 1 ||
        c->heads < 1 || (c->head_dim != 64 && c->head_dim != 128) ||
        (int64_t)c->pages * c->heads >= ((int64_t)1 << 31))  // (tensor maps count them in 32 bits)
        return FDLLM_ERR_ARG;
    int shift = 5;
    while (shift < 8 && (1 << shift) != c->page_size)
        ++shift;
    if ((1 << shift) != c->page_size)
        return FDLLM_ERR_ARG;
    for (const void *p : {c->k_codes, c->v_codes, c->k_affine, c->v_affine})
        if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0)
            return FDLLM_ERR_ALIGN;
    v.kc = static_cast<uint8_t *>(c->k_codes);
    v.vc = static_cast<uint8_t *>(c->v_codes);
    v.ka = static_cast<uint32_t *>(c->k_affine);
    v.va = static_cast<uint32_t *>(c->v_affine);
    v.pages = c->pages;
    v.heads = c->heads;
    v.page_shift = shift;
    v.D = c->head_dim;
    return FDLLM_OK;
}

// Slots of a block table are counted with 32 bits, and grids carry B and heads in y and z.
constexpr int kMaxGridYZ = 65535;
inline bool check_table(const int32_t *table, int B, int max_pages, int page_shift, int heads)
{
    return table && B >= 1 && B <= kMaxGridYZ && heads <= kMaxGridYZ && max_pages >= 1 &&
           ((int64_t)max_pages << page_shift) < ((int64_t)1 << 30);
}

// fdllm_cache_attention's and fdllm_cache_key_weights' queries (defined with the former).
bool check_queries(const void *q, const int64_t *strides, int dtype, int B, int Lq, int Hq,
                   int heads);

// The status word of the cache's kernels on the current device (null where it cannot be had);
// looked up once per device, so the first call on a device must not be under stream capture.
uint32_t *cache_status_word();

// A base and its strides as 16-byte vectors need them.
inline bool aligned16(const void *p, const int64_t *strides, int n, int esize)
{
    if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0)
        return false;
    for (int i = 0; i < n; ++i)
        if ((strides[i] * esize) % 16 != 0)
            return false;
    return true;
}

inline Strides3 strides3(const int64_t *s) { return Strides3{s[0], s[1], s[2]}; }

constexpr int kMaxCacheDevices = 64;

// What a kernel needs set up once on each device (its limit of shared memory holds for the
// current one only).  A failure is not kept: the next call tries again.  Two threads may come
// first at once; the set-up then runs twice, to the same end.
struct PerDevice {
    std::atomic<bool> ready[kMaxCacheDevices] = {};

    template <typename F>
    cudaError_t once(F setup)
    {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess)
            return e;
        if (dev < 0 || dev >= kMaxCacheDevices)
            return cudaErrorInvalidDevice;
        if (ready[dev].load(std::memory_order_acquire))
            return cudaSuccess;
        e = setup();
        if (e == cudaSuccess)
            ready[dev].store(true, std::memory_order_release);
        else
            cudaGetLastError();
        return e;
    }
};

// SMs of the current device (152, a GB300's, where there is none to ask).
inline int sm_count()
{
    static std::atomic<int> cached[kMaxCacheDevices] = {};
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxCacheDevices) {
        cudaGetLastError();
        return 152;
    }
    n = cached[dev].load(std::memory_order_relaxed);
    if (n > 0)
        return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 152;
    }
    cached[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Set on this thread while the decode loop (decode_loop.cu) captures its body without programmatic
// edges: the operators that a forward pass calls launch in plain stream order too.
extern thread_local bool plain_launches;

// One kernel launch; `pdl` makes it a programmatic dependent of the stream's previous kernel
// (the kernel then waits with pdl_wait() before it touches memory), but for plain_launches.
template <typename... P, typename... A>
cudaError_t launch(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream,
                   bool pdl, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl && !plain_launches ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, P(args)...);
}

#ifdef __CUDACC__

// Page holding slot `slot` of sequence b, or -1 where the table or the pool has none.
__device__ __forceinline__ int page_of(const CacheView &c, const int32_t *table, int max_pages,
                                       int b, int slot)
{
    const int i = slot >> c.page_shift;
    if (slot < 0 || i >= max_pages)
        return -1;
    const int pg = __ldg(table + (int64_t)b * max_pages + i);
    return (pg >= 0 && pg < c.pages) ? pg : -1;
}

// Index of (page, head, slot) into the affine arrays; times D/2, into k_codes.
__device__ __forceinline__ int64_t slot_index(const CacheView &c, int pg, int h, int slot)
{
    return (((int64_t)pg * c.heads + h) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
}

// Byte of v_codes holding channel d of (page, head, slot).
__device__ __forceinline__ int64_t v_byte(const CacheView &c, int pg, int h, int d, int slot)
{
    return ((((int64_t)pg * c.heads + h) * c.D + d) << (c.page_shift - 1)) +
           ((slot & ((1 << c.page_shift) - 1)) >> 1);
}

__device__ __forceinline__ float nan_f() { return __int_as_float(0x7FC00000); }
__device__ __forceinline__ float neg_inf_f() { return __int_as_float((int)0xFF800000); }

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <typename T>
__device__ __forceinline__ float to_float(T x);
template <>
__device__ __forceinline__ float to_float(float x) { return x; }
template <>
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float(float x) { return x; }
template <>
__device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }

// Eight consecutive values, 16-byte aligned.
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4 *>(p);
        const float4 b = *reinterpret_cast<const float4 *>(p + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
        x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 2 && __is_same(T, __nv_bfloat16)) {
                x[2 * i] = bf16_low(w[i]);
                x[2 * i + 1] = bf16_high(w[i]);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                x[2 * i] = f.x;
                x[2 * i + 1] = f.y;
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (__is_same(T, __nv_bfloat16)) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    } else {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *reinterpret_cast<uint4 *>(p) =
            make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]),
                       pack2<T>(x[6], x[7]));
    }
}

#endif  // __CUDACC__

}  // namespace fdllm
