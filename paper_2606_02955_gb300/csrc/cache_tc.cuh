// cache_tc.cuh -- tensor-core building blocks of the prefix cache's kernels: codes to matrix
// operands, the A operand in tensor memory, descriptors, packed arithmetic, column reductions
// and the tensor maps of a cache.
#pragma once

#include <cuda.h>

#include "cache.cuh"
#include "ptx.cuh"
#include "tcgen05.cuh"

namespace fdllm {

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                              const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                              const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeFn encode_tiled()
{
    static std::atomic<EncodeFn> encode{nullptr};
    if (const EncodeFn f = encode.load(std::memory_order_relaxed))
        return f;
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess) {
        cudaGetLastError();
        return nullptr;
    }
    encode.store(reinterpret_cast<EncodeFn>(p), std::memory_order_relaxed);
    return reinterpret_cast<EncodeFn>(p);
}

// One tensor map.  The driver's function wants the device's context current, which a host thread
// has only from its first runtime call that needs one on (memory a binding keeps needs none): a
// first failure makes it current and tries again.
inline bool encode_map(CUtensorMap *m, CUtensorMapDataType type, int rank, const void *base,
                       const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box,
                       CUtensorMapSwizzle swizzle, CUtensorMapL2promotion promotion)
{
    const EncodeFn encode = encode_tiled();
    const cuuint32_t unit[5] = {1, 1, 1, 1, 1};
    const auto done = [&] {
        return encode(m, type, (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, unit,
                      CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, promotion,
                      CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    if (!encode)
        return false;
    if (done())
        return true;
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess && done();
}

// Tensor map of rows [B, tokens, heads, D] of 16-bit values: one box `box_inner` channels of 32
// tokens of a head, swizzled where they are 64.  False where a map cannot hold the strides (an
// axis of several that repeats one row).
inline bool make_rows_map(CUtensorMap *m, const void *base, const Strides3 &s, int B, int tokens,
                          int heads, int D, int box_inner, bool swizzle)
{
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)tokens, (cuuint64_t)B};
    cuuint64_t strides[3];
    const int64_t elements[3] = {s.head, s.token, s.batch};
    for (int i = 0; i < 3; ++i) {
        const int64_t e = dims[i + 1] == 1 ? D : elements[i];
        if (e <= 0 || e >= ((int64_t)1 << 38))
            return false;
        strides[i] = 2 * (cuuint64_t)e;
    }
    const cuuint32_t box[4] = {(cuuint32_t)box_inner, 1, 32, 1};
    return encode_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, base, dims, strides, box,
                      swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_128B);
}

// Tensor maps of a cache's codes, with the page and head as an axis of its own (rows counted
// over all pages pass 31 bits in a pool of 73 GB): keys as rows of D/2 bytes, one box a page's (or
// a tile's) slots; values as rows of page/2 bytes, one box D channels of up to 128 slots.  The
// swizzle follows the box's row, so that 16-byte reads of one row a thread meet no bank twice.
inline bool make_cache_maps(const CacheView &c, CUtensorMap *k, CUtensorMap *v)
{
    const int page = 1 << c.page_shift, span = page < 128 ? page : 128;
    const auto map = [&](CUtensorMap *m, void *base, int inner, int rows, int box_inner,
                         int box_rows) {
        const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)rows,
                                    (cuuint64_t)c.pages * c.heads};
        const cuuint64_t strides[2] = {(cuuint64_t)inner, (cuuint64_t)inner * rows};
        const cuuint32_t box[3] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows, 1};
        const CUtensorMapSwizzle sw = box_inner == 64   ? CU_TENSOR_MAP_SWIZZLE_64B
                                      : box_inner == 32 ? CU_TENSOR_MAP_SWIZZLE_32B
                                                        : CU_TENSOR_MAP_SWIZZLE_NONE;
        return encode_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, base, dims, strides, box, sw,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
    };
    return map(k, c.kc, c.D / 2, page, c.D / 2, span) &&
           (!v || map(v, c.vc, page / 2, c.D, span / 2, c.D));
}

#ifdef __CUDACC__

__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, int32_t x, int32_t y,
                                            int32_t z, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_addr(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar))
        : "memory");
}

__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *map, int32_t x, int32_t y,
                                            int32_t z, int32_t w, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_addr(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_addr(bar))
        : "memory");
}

// ---------------------------------------------------------------- packed fp32 pairs
__device__ __forceinline__ uint64_t f2(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void un2(uint64_t v, float &lo, float &hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// Minima and maxima that are NaN where an argument is.
__device__ __forceinline__ float fmin_nan(float a, float b)
{
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float fmax_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

template <typename T>
__device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi)
{
    if constexpr (__is_same(T, __nv_bfloat16)) {
        lo = bf16_low(w);
        hi = bf16_high(w);
    } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
        lo = f.x;
        hi = f.y;
    }
}

// ---------------------------------------------------------------- codes -> matrix operands
// Inside every group of eight, the contraction runs over elements 0 4 1 5 2 6 3 7: the order in
// which masking a word of eight 4-bit codes yields pairs.
//
// A word's codes as four fp16 pairs, the codes of odd place 16 times as large; the other operand
// makes up for that.
//
// Keys: each code less 8.  A code in the lowest places of 1024 (fp16's unit there is 1) makes
// 1024 + code, or 1024 + 16 code, and 1032 or 1152 come off exactly.  Left where they lie, four
// bits are the subnormals code * 2^-24, for half the instructions; but the tensor core lines its
// products up by their exponents before it adds them, and subnormals lose as many places as they
// lack: scores were off by 5e-6, ten times what fp32 sums of the same terms are.
__device__ __forceinline__ void unpack32(const uint4 x, uint32_t (&y)[16])
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[4 * i] = (w[i] & 0x000F000Fu) | 0x64006400u;
        y[4 * i + 1] = (w[i] & 0x00F000F0u) | 0x64006400u;
        y[4 * i + 2] = ((w[i] >> 8) & 0x000F000Fu) | 0x64006400u;
        y[4 * i + 3] = ((w[i] >> 8) & 0x00F000F0u) | 0x64006400u;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(y[i]) : "r"(i & 1 ? 0x64806480u : 0x64086408u));
}

// Values: those subnormals (kSumUnit), since 5e-6 is a hundredth of what the results' types round;
// codes of odd place less 15, by their complement and the sign, so that sums over tens of thousands of keys do
// not grow to a multiple of what the offsets leave of them (of 32000 keys 2.4e-3 of the result;
// so 1.7e-3, which is what bf16 rounds).
__device__ __forceinline__ void unpack32_values(const uint4 x, uint32_t (&y)[16])
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[4 * i] = w[i] & 0x000F000Fu;
        y[4 * i + 1] = (~w[i] & 0x00F000F0u) | 0x80008000u;
        y[4 * i + 2] = (w[i] >> 8) & 0x000F000Fu;
        y[4 * i + 3] = (~(w[i] >> 8) & 0x00F000F0u) | 0x80008000u;
    }
}

// Eight 16-bit values in the same order.
__device__ __forceinline__ uint4 interleave8(const uint4 x)
{
    return make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632),
                      __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
}

// Queries against codes: fp16, times a power of two 2^-e that brings the row's largest to 2^13
// (0: 1), and 2^-4 in odd channels.  e from the largest; clamped so that 2^e and 2^-e exist.
__device__ __forceinline__ int query_exponent(float big)
{
    const int e = big > 0.0f ? (int)(__float_as_uint(big) >> 23) - 127 - 13 : 0;
    return min(max(e, -100), 100);
}

__device__ __forceinline__ float power_of_two(int e)  // of a normal number
{
    return __uint_as_float((uint32_t)(127 + e) << 23);
}

// Of eight channels of a query: their sum, and the largest finite one's size.
template <typename T>
__device__ __forceinline__ void sum_and_top(const uint4 x, float &sum, float &top)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    sum = top = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpack2<T>(w[i], lo, hi);
        sum += lo + hi;
        top = fmaxf(top, fabsf(lo) <= 3.4e38f ? fabsf(lo) : 0.0f);
        top = fmaxf(top, fabsf(hi) <= 3.4e38f ? fabsf(hi) : 0.0f);
    }
}

// Eight channels of a query, in the operand's order; unit = 2^-e.
template <typename T>
__device__ __forceinline__ uint4 code_queries(const uint4 x, float unit)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        unpack2<T>(w[i], f[2 * i], f[2 * i + 1]);
    const float odd = unit * 0.0625f;
    return make_uint4(pack2<__half>(f[0] * unit, f[4] * unit), pack2<__half>(f[1] * odd, f[5] * odd),
                      pack2<__half>(f[2] * unit, f[6] * unit), pack2<__half>(f[3] * odd, f[7] * odd));
}

// ---------------------------------------------------------------- tensor memory
// Columns of this warp's 32 lanes, one 32-bit word a column.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
        "%11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
        "r"(r[15])
        : "memory");
}

template <int NC>
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[NC])
{
    if constexpr (NC == 4) {
        asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr),
                     "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
                     : "memory");
    } else {
        static_assert(NC == 8, "columns");
        asm volatile(
            "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(
                taddr),
            "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]),
            "r"(r[7])
            : "memory");
    }
}

__device__ __forceinline__ void tmem_wait_st()
{
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

template <int NC>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[NC])
{
    if constexpr (NC == 16) {
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
            "%11, %12, %13, %14, %15}, [%16];"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
              "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
              "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
            : "r"(taddr)
            : "memory");
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                       "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                       "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                     :
                     : "memory");
    } else {
        static_assert(NC == 8, "columns");
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
              "=r"(r[7])
            : "r"(taddr)
            : "memory");
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                       "+r"(r[6]), "+r"(r[7])
                     :
                     : "memory");
    }
}

// ---------------------------------------------------------------- tcgen05.mma, A in tensor memory
// kind::f16 with fp32 accumulation: formats of A and B (both T), B K-major or (b_mn) with its
// rows contiguous (bit 16), N >> 3, M >> 4.
template <typename T>
__device__ __forceinline__ constexpr uint32_t idesc_f16(int M, int N, bool b_mn)
{
    const uint32_t f = __is_same(T, __nv_bfloat16) ? 1u : 0u;
    return (1u << 4) | (f << 7) | (f << 10) | (b_mn ? 1u << 16 : 0u) | (uint32_t(N >> 3) << 17) |
           (uint32_t(M >> 4) << 24);
}

// D[tmem] (+)= A[tmem] * B[smem] for one K = 16 slice, and a commit of all of them.  The whole
// warp calls these with the same operands and one lane of it issues: operands that the compiler
// knows to be uniform need no move of registers (N = 32: 17 cycles a product; issued under
// `if (lane == 0)` 47, whatever N).
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b32 x;\n\t"
        "elect.sync x|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void mma_commit(uint64_t *bar)
{
    asm volatile(
        "{\n\t.reg .pred e;\n\t.reg .b32 x;\n\t"
        "elect.sync x|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(
            smem_addr(bar))
        : "memory");
}

// Descriptor of an unswizzled operand with contiguous rows (MN-major): blocks of 8 rows x 8 k
// (a 16-byte line of 8 rows for each k, 128 bytes), `rows_step` bytes from a block to the next
// 8 rows, `k_step` bytes to the next 8 k.
__device__ __forceinline__ uint64_t mn_desc(const void *tile, uint32_t rows_step, uint32_t k_step)
{
    return (uint64_t)((smem_addr(tile) & 0x3FFFFu) >> 4) | ((uint64_t)(k_step >> 4) << 16) |
           ((uint64_t)(rows_step >> 4) << 32) | (1ull << 46);
}

// Shared-memory writes of this thread made visible to the tensor core.
__device__ __forceinline__ void fence_async_smem()
{
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// Waits on a shared-memory address, a few instructions each: many places of a kernel wait, and
// code that does not fit the instruction cache costs its warps more than the waits (with a timer at
// each place 64 blocks' attention took 195 us, then 143 without).  The limit is a count of tries; a
// try on a barrier that does not complete takes the hardware's 4 us (measured), so that 2^18 of
// them are a second, where a wait takes microseconds.
// kSleepNs: a warp that waits most of its time sleeps between tries, which would take issue slots
// from the warps that work.  False: given up; the caller waits no more, and says so in the status
// word.
constexpr uint32_t kWaitTries = 1u << 18, kDrainTries = 1u << 15;

__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}

template <int kSleepNs>
__device__ __forceinline__ bool mbar_wait_at(uint32_t bar, uint32_t parity,
                                             uint32_t tries = kWaitTries)
{
#pragma unroll 1
    for (uint32_t i = 0; i < tries; ++i) {
        if (mbar_try(bar, parity))
            return true;
        if constexpr (kSleepNs > 0)
            __nanosleep(kSleepNs);
    }
    return false;
}

// An arrival by the lanes where `who` holds (a predicate, not a branch).
__device__ __forceinline__ void mbar_arrive_if(uint32_t bar, bool who, uint32_t n = 1)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "@p mbarrier.arrive.shared::cta.b64 _, [%0], %2;\n\t}" ::"r"(bar),
        "r"((uint32_t)who), "r"(n)
        : "memory");
}

// Shared memory by address (a base kept in a register, not rebuilt at each use).
__device__ __forceinline__ float4 lds4f(uint32_t at)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(at)
                 : "memory");
    return v;
}
__device__ __forceinline__ uint4 lds4(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(at)
                 : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds1(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void sts4(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w)
                 : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Registers of the threads of a warpgroup, all of whose warps say so: given back, and taken of
// what the CTA's launch got for it (the groups' shares never add up to more than that).
template <int N>
__device__ __forceinline__ void reg_dec()
{
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void reg_inc()
{
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

// ---------------------------------------------------------------- barriers of some of a CTA's warps
__device__ __forceinline__ void named_sync(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

__device__ __forceinline__ bool named_sync_or(int id, int threads, bool x)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %3, 0;\n\t"
        "bar.red.or.pred q, %1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(id), "r"(threads), "r"((uint32_t)x)
        : "memory");
    return r != 0;
}

// Reduces each of NC columns over the warp's lanes: afterwards v[0] of lane c holds column
// c % NC.  NC - 1 shuffles, then one for each further halving of the lanes.
template <int NC, typename Op>
__device__ __forceinline__ void warp_columns(float (&v)[NC], Op op)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = NC / 2; h > 0; h >>= 1) {
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float send = (lane & h) ? v[i] : v[i + h];
            const float keep = (lane & h) ? v[i + h] : v[i];
            v[i] = op(keep, __shfl_xor_sync(0xFFFFFFFFu, send, h));
        }
    }
#pragma unroll
    for (int m = NC; m < 32; m <<= 1)
        v[0] = op(v[0], __shfl_xor_sync(0xFFFFFFFFu, v[0], m));
}

#endif  // __CUDACC__

}  // namespace fdllm
