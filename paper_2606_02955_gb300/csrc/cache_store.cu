// cache_store.cu -- fdllm_cache_append and fdllm_cache_read: rows of keys and values into the
// 4-bit prefix cache and back.
//
// Bound by memory: a row of D 16-bit values (2 D bytes) becomes D/2 bytes of codes and 4 bytes
// of scale and offset.
#include <cuda_runtime.h>

#include "cache.cuh"

namespace fdllm {
namespace {

// One CTA handles kSlots consecutive slots of one head, a piece that starts at a multiple of
// kSlots and so lies within one page: a thread holds 16 channels of one slot's keys and values,
// D / 16 lanes to a row.  The values' codes go through shared memory, because v_codes is
// channel-major: thread d then owns the 16 bytes of channel d.
constexpr int kSlots = 32;

struct StoreArgs {
    CacheView c;
    const int32_t *table;  // [B, max_pages]
    int max_pages;
    const int32_t *start;  // [B] or null
    const int32_t *count;  // [B] or null
    int n;
    const void *k;         // append: [B, n, heads, D]
    const void *v;
    Strides3 ks, vs;
    void *out_k;           // read: [B, n, heads, D]
    void *out_v;
};

__device__ __forceinline__ int count_of(const StoreArgs &a, int b)
{
    const int c = a.count ? a.count[b] : a.n;
    return min(max(c, 0), a.n);
}

// Scale and offset (packed) and the 16 codes (a byte each, four words) of this lane's part of
// a row of 16 * LANES values held by LANES neighbouring lanes.  All lanes of the warp take part.
template <int LANES>
__device__ __forceinline__ uint32_t quantise(const float (&x)[16], uint32_t (&codes)[4])
{
    float low = x[0], high = x[0], poison = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        low = fminf(low, x[i]);
        high = fmaxf(high, x[i]);
        poison = fmaf(x[i], 0.0f, poison);  // NaN from a NaN or an infinity
    }
#pragma unroll
    for (int m = LANES / 2; m > 0; m >>= 1) {
        low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, m));
        high = fmaxf(high, __shfl_xor_sync(0xFFFFFFFFu, high, m));
        poison += __shfl_xor_sync(0xFFFFFFFFu, poison, m);
    }
    const float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(__fsub_rn(high, low), 15.0f)));
    const float o = __bfloat162float(__float2bfloat16_rn(low));
    codes[0] = codes[1] = codes[2] = codes[3] = 0;
    if (!(fabsf(s) + fabsf(o) + poison < __int_as_float(0x7F800000)))
        return 0x7FC07FC0u;  // scale and offset NaN
    if (s != 0.0f) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float t = rintf(__fdiv_rn(__fsub_rn(x[i], o), s));
            codes[i >> 2] |= (uint32_t)fminf(fmaxf(t, 0.0f), 15.0f) << (8 * (i & 3));
        }
    }
    return (__float_as_uint(s) >> 16) | (__float_as_uint(o) & 0xFFFF0000u);
}

// Bytes of codes two to a word's low half -> nibbles: four byte codes -> 16 bits.
__device__ __forceinline__ uint32_t nibbles(uint32_t w)
{
    const uint32_t p = w | (w >> 4);  // byte 0: codes 0, 1; byte 2: codes 2, 3
    return (p & 0xFFu) | ((p >> 8) & 0xFF00u);
}

template <typename T, int D>
__global__ void __launch_bounds__(2 * D) append_kernel(const __grid_constant__ StoreArgs a)
{
    constexpr int kLanes = D / 16;
    __shared__ __align__(16) uint8_t vsm[kSlots][D];
    pdl_wait();
    const int h = blockIdx.y, b = blockIdx.z;
    const int start = a.start ? a.start[b] : 0;
    const int count = count_of(a, b);
    if (start < 0 || start > (a.max_pages << a.c.page_shift))
        return;
    const int slot0 = (start / kSlots + blockIdx.x) * kSlots;
    const int slot = slot0 + threadIdx.x / kLanes;
    const int part = threadIdx.x % kLanes;
    if (slot0 >= start + count)
        return;
    const int pg = page_of(a.c, a.table, a.max_pages, b, slot0);
    if (pg < 0)
        return;
    const int i = slot - start;
    const bool live = i >= 0 && i < count;
    float xk[16], xv[16];
#pragma unroll
    for (int j = 0; j < 16; ++j)
        xk[j] = xv[j] = 0.0f;
    if (live) {
        const T *k = static_cast<const T *>(a.k) + b * a.ks.batch + i * a.ks.token +
                     h * a.ks.head + 16 * part;
        const T *v = static_cast<const T *>(a.v) + b * a.vs.batch + i * a.vs.token +
                     h * a.vs.head + 16 * part;
        load8(k, reinterpret_cast<float (&)[8]>(xk[0]));
        load8(k + 8, reinterpret_cast<float (&)[8]>(xk[8]));
        load8(v, reinterpret_cast<float (&)[8]>(xv[0]));
        load8(v + 8, reinterpret_cast<float (&)[8]>(xv[8]));
    }
    uint32_t ck[4], cv[4];
    const uint32_t ak = quantise<kLanes>(xk, ck);
    const uint32_t av = quantise<kLanes>(xv, cv);
    const int64_t at = slot_index(a.c, pg, h, slot);
    if (live) {
        *reinterpret_cast<uint2 *>(a.c.kc + at * (D / 2) + 8 * part) =
            make_uint2(nibbles(ck[0]) | (nibbles(ck[1]) << 16),
                       nibbles(ck[2]) | (nibbles(ck[3]) << 16));
        if (part == 0) {
            a.c.ka[at] = ak;
            a.c.va[at] = av;
        }
    }
    *reinterpret_cast<uint4 *>(&vsm[slot - slot0][16 * part]) =
        make_uint4(cv[0], cv[1], cv[2], cv[3]);
    __syncthreads();
    const int d = threadIdx.x;
    if (d >= D)
        return;
    uint8_t *dst = a.c.vc + v_byte(a.c, pg, h, d, slot0);
    if (slot0 >= start && slot0 + kSlots <= start + count) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t x = 0;
#pragma unroll
            for (int t = 0; t < 8; ++t)
                x |= (uint32_t)vsm[8 * j + t][d] << (4 * t);
            w[j] = x;
        }
        *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
        return;
    }
    // A piece at the ends of the range: bytes that it fills by half keep their other slot.
    for (int j = 0; j < kSlots / 2; ++j) {
        const int s = slot0 + 2 * j;
        const bool lo = s >= start && s < start + count;
        const bool hi = s + 1 >= start && s + 1 < start + count;
        if (!lo && !hi)
            continue;
        uint8_t x = 0;
        if (!lo || !hi)
            x = dst[j] & (lo ? 0xF0u : 0x0Fu);
        if (lo)
            x |= vsm[2 * j][d];
        if (hi)
            x |= vsm[2 * j + 1][d] << 4;
        dst[j] = x;
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(2 * D) read_kernel(const __grid_constant__ StoreArgs a)
{
    constexpr int kLanes = D / 16;
    __shared__ __align__(16) uint8_t vsm[kSlots][D];
    pdl_wait();
    const int h = blockIdx.y, b = blockIdx.z;
    const int start = a.start ? a.start[b] : 0;
    const int count = count_of(a, b);
    // Token i of the call is slot start + i; the first piece starts at or before start.
    const int lead = ((start % kSlots) + kSlots) % kSlots;
    const int i0 = blockIdx.x * kSlots - lead;
    if (i0 >= a.n)
        return;
    const int i = i0 + threadIdx.x / kLanes;
    const int part = threadIdx.x % kLanes;
    // Slots are counted in 64 bits here: start is any int.
    const int64_t slot0 = (int64_t)start + i0;
    const bool inside = slot0 >= 0 && slot0 < ((int64_t)a.max_pages << a.c.page_shift);
    const int pg = inside ? page_of(a.c, a.table, a.max_pages, b, (int)slot0) : -1;
    const int s = inside ? (int)slot0 : 0;
    if (pg >= 0 && threadIdx.x < D) {
        const int d = threadIdx.x;
        const uint4 w = *reinterpret_cast<const uint4 *>(a.c.vc + v_byte(a.c, pg, h, d, s));
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < kSlots; ++j)
            vsm[j][d] = (x[j >> 3] >> (4 * (j & 7))) & 15u;
    }
    __syncthreads();
    if (i < 0 || i >= a.n)
        return;
    float xk[16], xv[16];
    if (i >= count) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            xk[j] = xv[j] = 0.0f;
    } else if (pg < 0) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            xk[j] = xv[j] = nan_f();
    } else {
        const int64_t at = slot_index(a.c, pg, h, s + threadIdx.x / kLanes);
        const uint2 w = *reinterpret_cast<const uint2 *>(a.c.kc + at * (D / 2) + 8 * part);
        const uint32_t ak = a.c.ka[at], av = a.c.va[at];
        const uint4 c = *reinterpret_cast<const uint4 *>(&vsm[threadIdx.x / kLanes][16 * part]);
        const uint32_t kw[2] = {w.x, w.y}, vw[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            xk[j] = fmaf(bf16_low(ak), (float)((kw[j >> 3] >> (4 * (j & 7))) & 15u),
                         bf16_high(ak));
            xv[j] = fmaf(bf16_low(av), (float)((vw[j >> 2] >> (8 * (j & 3))) & 15u),
                         bf16_high(av));
        }
    }
    const int64_t o = (((int64_t)b * a.n + i) * a.c.heads + h) * D + 16 * part;
    T *ok = static_cast<T *>(a.out_k) + o;
    T *ov = static_cast<T *>(a.out_v) + o;
    store8(ok, reinterpret_cast<float (&)[8]>(xk[0]));
    store8(ok + 8, reinterpret_cast<float (&)[8]>(xk[8]));
    store8(ov, reinterpret_cast<float (&)[8]>(xv[0]));
    store8(ov + 8, reinterpret_cast<float (&)[8]>(xv[8]));
}

// Pieces that n slots from any start can touch.
int pieces(int n) { return (int)(((int64_t)n + kSlots - 2) / kSlots + 1); }

template <typename T>
cudaError_t launch_append(const StoreArgs &a, int B, cudaStream_t s)
{
    const dim3 grid(pieces(a.n), a.c.heads, B);
    return a.c.D == 128 ? launch(append_kernel<T, 128>, grid, dim3(256), 0, s, true, a)
                        : launch(append_kernel<T, 64>, grid, dim3(128), 0, s, true, a);
}

template <typename T>
cudaError_t launch_read(const StoreArgs &a, int B, cudaStream_t s)
{
    const dim3 grid(pieces(a.n), a.c.heads, B);
    return a.c.D == 128 ? launch(read_kernel<T, 128>, grid, dim3(256), 0, s, true, a)
                        : launch(read_kernel<T, 64>, grid, dim3(128), 0, s, true, a);
}

bool valid_dtype(int d) { return d == FDLLM_BF16 || d == FDLLM_FP32 || d == FDLLM_FP16; }

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" {

fdllm_status fdllm_cache_append(const fdllm_cache *cache, const int32_t *block_table, int B,
                                int max_pages, const int32_t *start, const int32_t *count,
                                const void *k, const int64_t *k_strides, const void *v,
                                const int64_t *v_strides, int dtype, int n, void *stream)
{
    StoreArgs a = {};
    const fdllm_status st = check_cache(cache, a.c);
    if (st != FDLLM_OK)
        return st;
    if (!check_table(block_table, B, max_pages, a.c.page_shift, a.c.heads) ||
        !valid_dtype(dtype) || n < 0 || n >= (1 << 30) || !k_strides || !v_strides)
        return FDLLM_ERR_ARG;
    if (n == 0)
        return FDLLM_OK;
    if (!k || !v)
        return FDLLM_ERR_ARG;
    const int es = dtype == FDLLM_FP32 ? 4 : 2;
    if (!aligned16(k, k_strides, 3, es) || !aligned16(v, v_strides, 3, es))
        return FDLLM_ERR_ALIGN;
    a.table = block_table;
    a.max_pages = max_pages;
    a.start = start;
    a.count = count;
    a.n = n;
    a.k = k;
    a.v = v;
    a.ks = strides3(k_strides);
    a.vs = strides3(v_strides);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == FDLLM_BF16   ? launch_append<__nv_bfloat16>(a, B, s)
                          : dtype == FDLLM_FP16 ? launch_append<__half>(a, B, s)
                                                : launch_append<float>(a, B, s);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

fdllm_status fdllm_cache_read(const fdllm_cache *cache, const int32_t *block_table, int B,
                              int max_pages, const int32_t *start, const int32_t *count,
                              void *out_k, void *out_v, int dtype, int n, void *stream)
{
    StoreArgs a = {};
    const fdllm_status st = check_cache(cache, a.c);
    if (st != FDLLM_OK)
        return st;
    if (!check_table(block_table, B, max_pages, a.c.page_shift, a.c.heads) ||
        !valid_dtype(dtype) || n < 0 || n >= (1 << 30))
        return FDLLM_ERR_ARG;
    if (n == 0)
        return FDLLM_OK;
    if (!out_k || !out_v)
        return FDLLM_ERR_ARG;
    const int64_t none[1] = {0};
    if (!aligned16(out_k, none, 0, 1) || !aligned16(out_v, none, 0, 1))
        return FDLLM_ERR_ALIGN;
    a.table = block_table;
    a.max_pages = max_pages;
    a.start = start;
    a.count = count;
    a.n = n;
    a.out_k = out_k;
    a.out_v = out_v;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == FDLLM_BF16   ? launch_read<__nv_bfloat16>(a, B, s)
                          : dtype == FDLLM_FP16 ? launch_read<__half>(a, B, s)
                                                : launch_read<float>(a, B, s);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

}  // extern "C"
