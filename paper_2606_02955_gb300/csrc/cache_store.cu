// cache_store.cu -- fdllm_cache_append and fdllm_cache_read: rows of keys and values into the
// 4-bit prefix cache and back.
//
// Bound by memory: a row of D 16-bit values (2 D bytes) becomes D/2 bytes of codes and 4 bytes
// of scale and offset.
//
// Two forms.  A CTA of the tile form takes 32 slots of one head, so that a channel's values fill
// 16 bytes of v_codes: they change places (slot by channel to channel by slot) in registers and
// shared memory.  A few tokens would leave most of such a CTA idle: there 8 (D = 64: 4) lanes
// take two neighbouring slots, a byte of v_codes, and touch the bytes themselves.
//
// Measured: 8 sequences x 1021 rows of 32 heads of 128 channels, bf16 (169 MB moved each way):
// append 60 us (2.8 TB/s: the arithmetic of ranges and codes, and 32-byte pieces of pages of 64
// slots), read 34 us (5.0 TB/s).
#include <cuda_runtime.h>

#include <type_traits>

#include "cache.cuh"
#include "cache_tc.cuh"

namespace fdllm {
namespace {

constexpr int kSlots = 32;     // slots of a tile: a piece that lies within one page
// Calls of at most so many tokens take the few-token form.  64 sequences of 32 heads, append: of one
// token 7.1 us (tiles 10.8), of eight 11.5 (14.1), of sixteen 15.6 (15.7); read: of one 3.0 (5.3),
// of two 4.2 (5.5), of three 5.6 (5.5).
constexpr int kFewAppended = 8, kFewRead = 2;

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

// Sixteen values of this lane: smallest and largest, NaN where one of them is (an infinity makes
// the range one, or a NaN).  Values of 16 bits are compared two at a time.
template <typename T>
struct Row16 {
    uint32_t w[8];  // of 16-bit types, as they lie in memory
    __device__ __forceinline__ void load(const T *p)
    {
        const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            w[i] = 0;
    }
    __device__ __forceinline__ void two(int i, float &x, float &y) const
    {
        if constexpr (__is_same(T, __nv_bfloat16)) {
            x = bf16_low(w[i]);
            y = bf16_high(w[i]);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            x = f.x;
            y = f.y;
        }
    }
    __device__ __forceinline__ void range(float &low, float &high) const
    {
        using P = std::conditional_t<__is_same(T, __nv_bfloat16), __nv_bfloat162, __half2>;
        P lo = *reinterpret_cast<const P *>(&w[0]), hi = lo;
#pragma unroll
        for (int i = 1; i < 8; ++i) {
            const P x = *reinterpret_cast<const P *>(&w[i]);
            lo = __hmin2_nan(lo, x);
            hi = __hmax2_nan(hi, x);
        }
        low = fmin_nan(to_float(lo.x), to_float(lo.y));
        high = fmax_nan(to_float(hi.x), to_float(hi.y));
    }
};

template <>
struct Row16<float> {
    float v[16];
    __device__ __forceinline__ void load(const float *p)
    {
        load8(p, reinterpret_cast<float (&)[8]>(v[0]));
        load8(p + 8, reinterpret_cast<float (&)[8]>(v[8]));
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            v[i] = 0.0f;
    }
    __device__ __forceinline__ void two(int i, float &x, float &y) const
    {
        x = v[2 * i];
        y = v[2 * i + 1];
    }
    __device__ __forceinline__ void range(float &low, float &high) const
    {
        low = high = v[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) {
            low = fmin_nan(low, v[i]);
            high = fmax_nan(high, v[i]);
        }
    }
};

// (x - o) / s, rounded to the nearest integer (ties to even) and clamped to 0..15, as bytes;
// `near` becomes the largest distance of a quotient from its integer.  15 sat(d / (15 s)) clamps
// in the product; adding 1.5 * 2^23 rounds.
constexpr float kMagic = 12582912.0f;

template <bool kExact, typename T>
__device__ __forceinline__ void round_codes(const Row16<T> &x, float o, float s, float inv15,
                                            uint32_t (&codes)[4], float &near)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x0, x1, t0, t1;
            x.two(2 * i + e, x0, x1);
            if constexpr (kExact) {
                t0 = __saturatef(__fdiv_rn(__fsub_rn(x0, o), s) * (1.0f / 16.0f));
                t1 = __saturatef(__fdiv_rn(__fsub_rn(x1, o), s) * (1.0f / 16.0f));
                u[2 * e] = __float_as_uint(__fadd_rn(fminf(t0 * 16.0f, 15.0f), kMagic));
                u[2 * e + 1] = __float_as_uint(__fadd_rn(fminf(t1 * 16.0f, 15.0f), kMagic));
            } else {
                un2(add2(f2(x0, x1), f2(-o, -o)), t0, t1);
                t0 = __saturatef(t0 * inv15);
                t1 = __saturatef(t1 * inv15);
                const uint64_t t = f2(t0, t1);
                const uint64_t r = fma2(t, f2(15.0f, 15.0f), f2(kMagic, kMagic));
                const uint64_t q = add2(r, f2(-kMagic, -kMagic));
                float e0, e1, r0, r1;
                un2(fma2(t, f2(-15.0f, -15.0f), q), e0, e1);
                un2(r, r0, r1);
                near = max3(near, fabsf(e0), fabsf(e1));
                u[2 * e] = __float_as_uint(r0);
                u[2 * e + 1] = __float_as_uint(r1);
            }
        }
        codes[i] = __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040),
                               0x5410);
    }
}

// Scale and offset (packed) and the 16 codes (a byte each, four words) of this lane's part of
// a row of 16 * LANES values held by LANES neighbouring lanes.  All lanes of the warp take part.
template <int LANES, typename T>
__device__ __forceinline__ uint32_t quantise(const Row16<T> &x, uint32_t (&codes)[4])
{
    float low, high;
    x.range(low, high);
#pragma unroll
    for (int m = LANES / 2; m > 0; m >>= 1) {
        low = fmin_nan(low, __shfl_xor_sync(0xFFFFFFFFu, low, m));
        high = fmax_nan(high, __shfl_xor_sync(0xFFFFFFFFu, high, m));
    }
    const float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(__fsub_rn(high, low), 15.0f)));
    const float o = __bfloat162float(__float2bfloat16_rn(low));
    codes[0] = codes[1] = codes[2] = codes[3] = 0;
    if (!(fabsf(s) + fabsf(o) < __int_as_float(0x7F800000)))
        return 0x7FC07FC0u;  // scale and offset NaN
    if (s != 0.0f) {
        // The product with the reciprocal is within 2^-21 of the quotient, relatively (2^-17 of
        // 15): only where it comes that close to a half can the two round differently, and there
        // (or with a reciprocal that is not a normal number) the division decides.
        const float inv15 = __fdiv_rn(1.0f / 15.0f, s);
        float near = 0.0f;
        const bool normal = s > 0x1p-110f && s < 0x1p110f;
        round_codes<false>(x, o, s, inv15, codes, near);
        if (!normal || near > 0.49998f)
            round_codes<true>(x, o, s, inv15, codes, near);
    }
    return (__float_as_uint(s) >> 16) | (__float_as_uint(o) & 0xFFFF0000u);
}

// Bytes of codes -> nibbles: four byte codes -> 16 bits.
__device__ __forceinline__ uint32_t nibbles(uint32_t w)
{
    const uint32_t p = w | (w >> 4);  // byte 0: codes 0, 1; byte 2: codes 2, 3
    return (p & 0xFFu) | ((p >> 8) & 0xFF00u);
}

// A row's codes of this lane as 8 bytes of k_codes.
__device__ __forceinline__ uint2 row_nibbles(const uint32_t (&c)[4])
{
    return make_uint2(nibbles(c[0]) | (nibbles(c[1]) << 16), nibbles(c[2]) | (nibbles(c[3]) << 16));
}

template <typename T>
__device__ __forceinline__ void store16(T *p, const float (&x)[16])
{
    store8(p, reinterpret_cast<const float (&)[8]>(x[0]));
    store8(p + 8, reinterpret_cast<const float (&)[8]>(x[8]));
}

template <typename T>
__device__ __forceinline__ const T *row_of(const void *p, const Strides3 &s, int b, int i, int h)
{
    return static_cast<const T *>(p) + b * s.batch + i * s.token + h * s.head;
}

// Code `c` (an integer below 16) of a row with this scale and offset.
__device__ __forceinline__ float value_of(uint32_t c, uint32_t affine)
{
    return fmaf(bf16_low(affine), __uint_as_float(c | 0x4B000000u) - 8388608.0f,
                bf16_high(affine));
}

// The tile form.  A thread holds 16 channels of one slot, kLanes = D / 16 lanes a row.
template <typename T, int D>
__global__ void __launch_bounds__(2 * D) append_kernel(const __grid_constant__ StoreArgs a)
{
    constexpr int kLanes = D / 16;
    __shared__ __align__(16) uint16_t quad[kSlots / 4][D];  // four slots of a channel
    pdl_wait();
    const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 31;
    const int start = a.start ? a.start[b] : 0;
    const int count = count_of(a, b);
    if (start < 0 || start > (a.max_pages << a.c.page_shift))
        return;
    const int slot0 = (start / kSlots + blockIdx.x) * kSlots;
    const int slot = slot0 + threadIdx.x / kLanes;
    const int part = threadIdx.x % kLanes;
    if (slot0 >= start + count)
        return;
    // (the page is looked up while the rows are on their way)
    const int i = slot - start;
    const bool live = i >= 0 && i < count;
    Row16<T> xk, xv;
    xk.clear();
    xv.clear();
    if (live) {
        xk.load(row_of<T>(a.k, a.ks, b, i, h) + 16 * part);
        xv.load(row_of<T>(a.v, a.vs, b, i, h) + 16 * part);
    }
    const int pg = page_of(a.c, a.table, a.max_pages, b, slot0);
    if (pg < 0)
        return;
    uint32_t c[4];
    const int64_t at = slot_index(a.c, pg, h, slot);
    const uint32_t ak = quantise<kLanes>(xk, c);
    if (live)
        *reinterpret_cast<uint2 *>(a.c.kc + at * (D / 2) + 8 * part) = row_nibbles(c);
    const uint32_t av = quantise<kLanes>(xv, c);
    if (live && part == 0) {
        a.c.ka[at] = ak;
        a.c.va[at] = av;
    }
    // Two slots to a byte: the even slot's lane takes the lower eight channels of both, the odd
    // slot's the upper; then four slots to 16 bits, four channels a lane.
    const bool odd = lane & kLanes, high = lane & (2 * kLanes);
    uint32_t p[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t mine = odd ? c[2 + e] : c[e], give = odd ? c[e] : c[2 + e];
        const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, give, kLanes);
        p[e] = odd ? got | (mine << 4) : mine | (got << 4);
    }
    const uint32_t mine = high ? p[1] : p[0];
    const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, high ? p[0] : p[1], 2 * kLanes);
    const uint32_t lo = high ? got : mine, hi = high ? mine : got;  // slots 0, 1; slots 2, 3
    const int channel = 16 * part + (odd ? 8 : 0) + (high ? 4 : 0);
    *reinterpret_cast<uint2 *>(&quad[(slot - slot0) / 4][channel]) =
        make_uint2(__byte_perm(lo, hi, 0x5140), __byte_perm(lo, hi, 0x7362));
    __syncthreads();
    const int d = threadIdx.x;
    if (d >= D)
        return;
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        w[j] = quad[2 * j][d] | ((uint32_t)quad[2 * j + 1][d] << 16);
    uint4 *dst = reinterpret_cast<uint4 *>(a.c.vc + v_byte(a.c, pg, h, d, slot0));
    const int first = max(start - slot0, 0), last = min(start + count - slot0, kSlots);
    if (first > 0 || last < kSlots) {
        // A piece at the ends of the range keeps the slots that the call does not write.
        const uint4 was = *dst;
        const uint32_t o[4] = {was.x, was.y, was.z, was.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int from = min(max(first - 8 * j, 0), 8), to = min(max(last - 8 * j, 0), 8);
            const uint64_t all = (1ull << (4 * to)) - 1, none = (1ull << (4 * from)) - 1;
            const uint32_t m = to > from ? (uint32_t)(all & ~none) : 0u;
            w[j] = (w[j] & m) | (o[j] & ~m);
        }
    }
    *dst = make_uint4(w[0], w[1], w[2], w[3]);
}

// Reading goes from the page to the codes to the rows; kReadTiles tiles of a CTA make that way
// together.
constexpr int kReadTiles = 2;

template <typename T, int D>
__global__ void __launch_bounds__(2 * D) read_kernel(const __grid_constant__ StoreArgs a)
{
    constexpr int kLanes = D / 16;
    __shared__ __align__(16) uint16_t quad[kReadTiles][kSlots / 4][D];
    pdl_wait();
    const int h = blockIdx.y, b = blockIdx.z;
    const int start = a.start ? a.start[b] : 0;
    const int count = count_of(a, b);
    // Token i of the call is slot start + i; the first piece starts at or before start.
    const int lead = ((start % kSlots) + kSlots) % kSlots;
    const int64_t i00 = (int64_t)blockIdx.x * kReadTiles * kSlots - lead;
    if (i00 >= a.n)
        return;
    const int in = threadIdx.x / kLanes, part = threadIdx.x % kLanes;
    int pg[kReadTiles], s[kReadTiles];
#pragma unroll
    for (int t = 0; t < kReadTiles; ++t) {
        const int64_t i0 = i00 + t * kSlots, slot0 = start + i0;
        const bool inside = slot0 >= 0 && slot0 < ((int64_t)a.max_pages << a.c.page_shift);
        s[t] = inside ? (int)slot0 : 0;
        pg[t] = inside && i0 < count ? page_of(a.c, a.table, a.max_pages, b, s[t]) : -1;
    }
    uint2 kw[kReadTiles];
    uint32_t ak[kReadTiles], av[kReadTiles];
    uint4 w[kReadTiles];
    bool live[kReadTiles];
#pragma unroll
    for (int t = 0; t < kReadTiles; ++t) {
        const int64_t i = i00 + t * kSlots + in;
        live[t] = i >= 0 && i < count && pg[t] >= 0;
        kw[t] = make_uint2(0, 0);
        ak[t] = av[t] = 0;
        w[t] = make_uint4(0, 0, 0, 0);
        if (live[t]) {
            const int64_t at = slot_index(a.c, pg[t], h, s[t] + in);
            kw[t] = *reinterpret_cast<const uint2 *>(a.c.kc + at * (D / 2) + 8 * part);
            ak[t] = a.c.ka[at];
            av[t] = a.c.va[at];
        }
        if (pg[t] >= 0 && threadIdx.x < D)
            w[t] = *reinterpret_cast<const uint4 *>(a.c.vc +
                                                    v_byte(a.c, pg[t], h, threadIdx.x, s[t]));
    }
    if (threadIdx.x < D) {
#pragma unroll
        for (int t = 0; t < kReadTiles; ++t) {
            const uint32_t x[4] = {w[t].x, w[t].y, w[t].z, w[t].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                quad[t][2 * j][threadIdx.x] = (uint16_t)x[j];
                quad[t][2 * j + 1][threadIdx.x] = (uint16_t)(x[j] >> 16);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kReadTiles; ++t) {
        const int64_t i = i00 + t * kSlots + in;
        if (i < 0 || i >= a.n)
            continue;
        const int64_t o = (((int64_t)b * a.n + i) * a.c.heads + h) * D + 16 * part;
        T *ok = static_cast<T *>(a.out_k) + o;
        T *ov = static_cast<T *>(a.out_v) + o;
        float x[16];
        if (!live[t]) {
            // behind the count: 0; no such slot: NaN
#pragma unroll
            for (int j = 0; j < 16; ++j)
                x[j] = i >= count ? 0.0f : nan_f();
            store16(ok, x);
            store16(ov, x);
            continue;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j)
            x[j] = value_of(((j < 8 ? kw[t].x : kw[t].y) >> (4 * (j & 7))) & 15u, ak[t]);
        store16(ok, x);
        const uint4 *q = reinterpret_cast<const uint4 *>(&quad[t][in / 4][16 * part]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint4 v = q[j];
            const uint32_t c[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t two = c[e] >> (4 * (in & 3));  // this slot's codes of two channels
                x[8 * j + 2 * e] = value_of(two & 15u, av[t]);
                x[8 * j + 2 * e + 1] = value_of((two >> 16) & 15u, av[t]);
            }
        }
        store16(ov, x);
    }
}

// The few-token form: kLanes lanes a pair of slots (2 m, 2 m + 1) of one head.
template <typename T, int D>
__global__ void __launch_bounds__(128) append_few_kernel(const __grid_constant__ StoreArgs a,
                                                         int pairs)
{
    constexpr int kLanes = D / 16;
    pdl_wait();
    const int b = blockIdx.y, part = threadIdx.x % kLanes;
    const int row = (blockIdx.x * 128 + threadIdx.x) / kLanes;  // head * pairs + pair
    const int h = row / pairs, pair = row - h * pairs;
    const int start = a.start ? a.start[b] : 0;
    const int end = start + count_of(a, b);
    const bool there = h < a.c.heads && start >= 0 && start <= (a.max_pages << a.c.page_shift);
    const int slot0 = there ? (start / 2 + pair) * 2 : 0;
    const int pg = there && slot0 < end ? page_of(a.c, a.table, a.max_pages, b, slot0) : -1;
    uint32_t cv[2][4];
    bool live[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int slot = slot0 + e, i = slot - start;
        live[e] = pg >= 0 && slot >= start && slot < end;
        Row16<T> xk, xv;
        xk.clear();
        xv.clear();
        if (live[e]) {
            xk.load(row_of<T>(a.k, a.ks, b, i, h) + 16 * part);
            xv.load(row_of<T>(a.v, a.vs, b, i, h) + 16 * part);
        }
        uint32_t ck[4];
        const uint32_t ak = quantise<kLanes>(xk, ck);
        const uint32_t av = quantise<kLanes>(xv, cv[e]);
        if (live[e]) {
            const int64_t at = slot_index(a.c, pg, h, slot);
            *reinterpret_cast<uint2 *>(a.c.kc + at * (D / 2) + 8 * part) = row_nibbles(ck);
            if (part == 0) {
                a.c.ka[at] = ak;
                a.c.va[at] = av;
            }
        }
    }
    if (!live[0] && !live[1])
        return;
    uint8_t *v = a.c.vc + v_byte(a.c, pg, h, 16 * part, slot0);
    const int64_t step = (int64_t)1 << (a.c.page_shift - 1);  // a channel to the next
    const uint32_t keep = live[0] && live[1] ? 0u : live[0] ? 0xF0u : 0x0Fu;
    uint32_t old[16];
#pragma unroll
    for (int j = 0; j < 16; ++j)
        old[j] = keep ? v[j * step] : 0u;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const uint32_t lo = (cv[0][j >> 2] >> (8 * (j & 3))) & 15u;
        const uint32_t hi = (cv[1][j >> 2] >> (8 * (j & 3))) & 15u;
        v[j * step] = (uint8_t)((old[j] & keep) | ((lo | (hi << 4)) & ~keep));
    }
}

// kLanes lanes a token of one head.
template <typename T, int D>
__global__ void __launch_bounds__(128) read_few_kernel(const __grid_constant__ StoreArgs a)
{
    constexpr int kLanes = D / 16;
    pdl_wait();
    const int b = blockIdx.y, part = threadIdx.x % kLanes;
    const int row = (blockIdx.x * 128 + threadIdx.x) / kLanes;  // token * heads + head
    const int i = row / a.c.heads, h = row - i * a.c.heads;
    if (i >= a.n)
        return;
    const int64_t slot = (int64_t)(a.start ? a.start[b] : 0) + i;
    const int count = count_of(a, b);
    const bool inside = slot >= 0 && slot < ((int64_t)a.max_pages << a.c.page_shift);
    const int pg = inside && i < count ? page_of(a.c, a.table, a.max_pages, b, (int)slot) : -1;
    const int64_t o = (((int64_t)b * a.n + i) * a.c.heads + h) * D + 16 * part;
    float xk[16], xv[16];
#pragma unroll
    for (int j = 0; j < 16; ++j)
        xk[j] = xv[j] = i >= count ? 0.0f : nan_f();
    if (pg >= 0) {
        const int64_t at = slot_index(a.c, pg, h, (int)slot);
        const uint8_t *v = a.c.vc + v_byte(a.c, pg, h, 16 * part, (int)slot);
        const int64_t step = (int64_t)1 << (a.c.page_shift - 1);
        const uint2 kw = *reinterpret_cast<const uint2 *>(a.c.kc + at * (D / 2) + 8 * part);
        uint32_t c[16];
#pragma unroll
        for (int j = 0; j < 16; ++j)
            c[j] = v[j * step];
        const uint32_t ak = a.c.ka[at], av = a.c.va[at];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            xk[j] = value_of(((j < 8 ? kw.x : kw.y) >> (4 * (j & 7))) & 15u, ak);
            xv[j] = value_of((c[j] >> (4 * ((int)slot & 1))) & 15u, av);
        }
    }
    store16(static_cast<T *>(a.out_k) + o, xk);
    store16(static_cast<T *>(a.out_v) + o, xv);
}

// Pieces that n slots from any start can touch.
int pieces(int n) { return (int)(((int64_t)n + kSlots - 2) / kSlots + 1); }

template <typename T, int D>
cudaError_t launch_append_rows(const StoreArgs &a, int B, cudaStream_t s)
{
    if (a.n <= kFewAppended) {
        const int pairs = a.n / 2 + 1;
        const unsigned blocks = (unsigned)(((int64_t)a.c.heads * pairs * (D / 16) + 127) / 128);
        return launch(append_few_kernel<T, D>, dim3(blocks, B), dim3(128), 0, s, true, a, pairs);
    }
    return launch(append_kernel<T, D>, dim3(pieces(a.n), a.c.heads, B), dim3(2 * D), 0, s, true, a);
}

template <typename T, int D>
cudaError_t launch_read_rows(const StoreArgs &a, int B, cudaStream_t s)
{
    if (a.n <= kFewRead) {
        const unsigned blocks = (unsigned)(((int64_t)a.c.heads * a.n * (D / 16) + 127) / 128);
        return launch(read_few_kernel<T, D>, dim3(blocks, B), dim3(128), 0, s, true, a);
    }
    return launch(read_kernel<T, D>,
                  dim3((pieces(a.n) + kReadTiles - 1) / kReadTiles, a.c.heads, B), dim3(2 * D), 0, s, true, a);
}

template <typename T>
cudaError_t launch_append(const StoreArgs &a, int B, cudaStream_t s)
{
    return a.c.D == 128 ? launch_append_rows<T, 128>(a, B, s) : launch_append_rows<T, 64>(a, B, s);
}

template <typename T>
cudaError_t launch_read(const StoreArgs &a, int B, cudaStream_t s)
{
    return a.c.D == 128 ? launch_read_rows<T, 128>(a, B, s) : launch_read_rows<T, 64>(a, B, s);
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
