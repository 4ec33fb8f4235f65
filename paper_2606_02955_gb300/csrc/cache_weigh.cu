// cache_weigh.cu -- fdllm_cache_key_weights: the attention that each cached key receives, on the
// fifth-generation tensor cores.
//
// w_j += sum over the rows r (queries x heads of the group) of e^(s_rj - lse_r), with the scores
// of cache_attention.cu: s_rj = scale (ks_j (q_r . u_j) + ko_j sum(q_r)).
//
// Layout.  A tile is 128 keys.  S^T [128 keys x N rows] = K . Q^T puts a key's scores in one
// thread, so that the sum over the rows never leaves it: no shuffle, no atomic, one order.  The
// unpacked keys stay in tensor memory while the row tiles of a group (four of 64 rows, their
// queries in shared memory) pass by; more rows take the CTA's keys once again.
//
// Bound by the scores' arithmetic and the exponentials (a warpgroup of two weighs, the other only
// unpacks) above about 32 rows a head, below that by the codes: D/2 + 4 bytes of the cache a key, and 8 of weights.
//
// Split.  The key tiles of all (sequence, head) units in order are cut into equal ranges, one to
// a CTA; tiles share nothing, so nothing is joined.
//
// Measured (GPU time, each launch by itself): 8 sequences of 32 queries over 500 to 1024 keys, 32
// heads of 128 channels: 16 us; 2 sequences of 64 queries of 32 heads over 32000 keys of 8 (256 rows a
// head): 68 (calls in a row: 65).
#include <cuda_runtime.h>

#include <type_traits>

#include "cache.cuh"
#include "cache_tc.cuh"

namespace fdllm {
namespace {

constexpr int kKeys = 128;   // keys of a tile
constexpr float kLog2eLow = 1.925963e-08f;  // log2(e) - kLog2e
constexpr int kUnitCost = 1; // a segment's queries cost about as much as this many tiles

struct WeighArgs {
    CacheView c;
    const int32_t *table;
    int max_pages;
    const int32_t *lens;
    const void *q;
    Strides3 qs;
    int B, Lq, Hq, group;
    const float *lse;         // [B, Lq, Hq]
    float scale;              // times log2(e)
    const float *in;          // [B, heads, max_len] or null
    float *out;
    int max_len;
    int rows;                 // Lq * group
    uint32_t *status;         // sticky: a bounded wait gave up
};

template <int D_, int N_>
struct Shape {
    static constexpr int D = D_;
    static constexpr int N = N_;                    // rows of a row tile
    static constexpr int group = N >= 64 ? 4 : 1;   // row tiles whose queries are held
    static constexpr int loader = 8, issuer = 9;    // warps 0-3 unpack, 4-7 weigh
    static constexpr int threads = 320;
    static constexpr int ctas = 2;                  // CTAs an SM holds
    static constexpr int stages = 4;
    static constexpr int code_bytes = kKeys * D / 2;
    static constexpr int stage_bytes = code_bytes + 1024;  // (512 of it scales and offsets)
    static constexpr int q_off = stages * stage_bytes;
    static constexpr int q_bytes = N * D * 2;       // of a row tile
    static constexpr int smem = q_off + group * q_bytes + 1024;
    static constexpr int tK = 0, tS = 64;
    static constexpr int tmem = tS + 2 * N <= 128 ? 128 : 256;
    static_assert(tS + 2 * N <= tmem && ctas * tmem <= 512, "tensor memory");
};

// A sequence's cached length, or -1 where it is out of range.
__device__ __forceinline__ int length_of(const WeighArgs &a, int b)
{
    const int n = a.lens[b];
    return n >= 0 && n <= (a.max_pages << a.c.page_shift) && n <= a.max_len ? n : -1;
}

// Places of one unit in the call's order: its tiles and the charge for its beginning.
__device__ __forceinline__ int places_of(int n)
{
    return n > 0 ? (n + kKeys - 1) / kKeys + kUnitCost : 0;
}

template <typename S, typename T>
__global__ void __launch_bounds__(S::threads, S::ctas)
    weigh_kernel(const __grid_constant__ WeighArgs a, const __grid_constant__ CUtensorMap k_map)
{
    constexpr int D = S::D, N = S::N;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    // Memory barriers: the ring's stages full and empty; scores done, by their parity; all of a
    // key tile's products done, its keys unpacked; scores read, by their parity.  (Each is waited
    // for phase by phase: a wait two phases ahead would take the phase before last for its own.)
    enum { kFull = 0, kEmpty = kFull + S::stages, kSDone = kEmpty + S::stages,
           kKFree = kSDone + 2, kKReady, kSFree, kBars = kSFree + 2 };
    enum { kBarW = 1 };  // CTA barrier of the unpacking and weighing warps
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ uint32_t tmem_base;
    __shared__ uint8_t bad_pieces[S::stages];   // pieces of a stage's tile whose page is out of range
    __shared__ int64_t scan[S::threads / 32];
    __shared__ int64_t find_base;
    __shared__ int find_b;
    // of the queries held: sum of the channels; their unit; -lse in base 2 (-inf: the row counts
    // nothing)
    __shared__ __align__(16) float sumq[S::group * N], mulq[S::group * N], nlse[S::group * N];

    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i)
            mbar_init(&bars[i], i >= kEmpty && i < kSDone ? 8 : i >= kKReady ? 4 : 1);
        fence_mbar_init();
    }
    if (warp == S::issuer)
        tc::tmem_alloc(&tmem_base, S::tmem);
    pdl_wait();

    // The call's places and the sequence in which this CTA's range begins.
    int64_t at, end, base = 0;
    int b = 0;
    {
        const int run = (a.B + S::threads - 1) / S::threads;
        const int b0 = min(a.B, tid * run), b1 = min(a.B, b0 + run);
        int64_t mine = 0;
        for (int i = b0; i < b1; ++i)
            mine += places_of(length_of(a, i));
        int64_t upto = mine;
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const int64_t o = __shfl_up_sync(0xFFFFFFFFu, upto, m);
            upto += lane >= m ? o : 0;
        }
        if (lane == 31)
            scan[warp] = upto;
        __syncthreads();
        int64_t before = 0, total = 0;
        for (int i = 0; i < S::threads / 32; ++i) {
            before += i < warp ? scan[i] : 0;
            total += scan[i];
        }
        total *= a.c.heads;
        const int64_t p0 = (before + upto - mine) * a.c.heads;
        at = total * blockIdx.x / gridDim.x;
        end = total * (blockIdx.x + 1) / gridDim.x;
        if (mine > 0 && at >= p0 && at < p0 + mine * a.c.heads) {
            find_base = p0;
            find_b = b0;
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tmem_base, 0);
    if (at < end) {
        base = find_base;
        b = find_b;
    }
    pdl_launch_dependents();

    uint32_t bar0 = smem_addr(bars), buf0 = smem_addr(smem), sum0 = smem_addr(sumq),
             mul0 = smem_addr(mulq), lse0 = smem_addr(nlse);
    asm volatile("" : "+r"(bar0), "+r"(buf0), "+r"(sum0), "+r"(mul0), "+r"(lse0));
    auto bar = [&](int i) { return bar0 + 8u * i; };
    // A wait gave up: no further wait.  The loading and the issuing warp stop at once and wait, with
    // a limit, for what they have in flight; the others walk on to the end of their range.
    bool dead = false;
    auto wait = [&](auto sleep, int i, uint32_t parity) {
        if (!dead && !mbar_wait_at<decltype(sleep)::value>(bar(i), parity))
            dead = true;
    };
    using Long = std::integral_constant<int, 100>;
    using Short = std::integral_constant<int, 20>;
    using Now = std::integral_constant<int, 0>;

    // The CTA's range, segment by segment: tiles [first, last) of (b, h), and for each group of
    // row tiles [g0, g0 + rows_held) once.  All warps walk it alike.
    int h = 0, first = 0, last = 0, n = 0;
    auto next = [&]() -> bool {
        while (at < end) {
            n = length_of(a, b);
            int len = places_of(n);
            while (at >= base + (int64_t)len * a.c.heads) {
                base += (int64_t)len * a.c.heads;
                n = length_of(a, ++b);
                len = places_of(n);
            }
            const int64_t local = at - base;
            h = (int)(local / len);
            const int from = (int)(local - (int64_t)h * len);
            const int to = (int)min((int64_t)len, from + (end - at));
            at += to - from;
            first = min(from, len - kUnitCost);
            last = min(to, len - kUnitCost);
            if (first < last)
                return true;
        }
        return false;
    };
    constexpr int kHeld = S::group * N;

    // Rows [g0, g0 + held) of the queries into the operand, by the unpacking and the weighing
    // warps together: times a power of two of each row, with their sums in that unit.  Their -lse
    // lose the whole number `shift`, near all of them as a rule, so that the small differences of
    // large scores keep their bits.
    // A row whose -lse is infinite counts nothing, whatever it holds: its queries are taken as 0.
    auto hold_queries = [&](int g0, int held, float &shift) {
        const auto lse_of = [&](int r) {
            const int qi = (g0 + r) / a.group, g = (g0 + r) - qi * a.group;
            return a.lse[((int64_t)b * a.Lq + qi) * a.Hq + h * a.group + g];
        };
        const int chunks = (held + N - 1) / N * N * (D / 8);  // of 8 channels
        named_sync(kBarW, 256);
#pragma unroll 4
        for (int i = tid; i < chunks; i += 256) {
            const int r = i / (D / 8), c8 = i % (D / 8), m = r % N;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (r < held) {
                const int qi = (g0 + r) / a.group, g = (g0 + r) - qi * a.group;
                x = *reinterpret_cast<const uint4 *>(
                    static_cast<const T *>(a.q) + b * a.qs.batch + qi * a.qs.token +
                    (int64_t)(h * a.group + g) * a.qs.head + 8 * c8);
                if (lse_of(r) == neg_inf_f())
                    x = make_uint4(0, 0, 0, 0);
            }
            float sum, top;
            sum_and_top<T>(x, sum, top);
#pragma unroll
            for (int s = D / 16; s > 0; s >>= 1) {
                sum += __shfl_xor_sync(0xFFFFFFFFu, sum, s);
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
            }
            const int e = query_exponent(top);
            const float unit = power_of_two(-e);
            if (c8 == 0) {
                sumq[r] = sum * unit;
                mulq[r] = power_of_two(e);
            }
            *reinterpret_cast<uint4 *>(smem + S::q_off + r / N * S::q_bytes + (c8 >> 3) * (N * 128) +
                                       m * 128 + (((c8 & 7) ^ (m & 7)) << 4)) =
                code_queries<T>(x, unit);
        }
        const float l0 = lse_of(0);
        shift = fabsf(l0) < 1e6f ? rintf(-l0 * kLog2e) : 0.0f;
        for (int r = tid; r < kHeld; r += 256) {
            float x = neg_inf_f();
            if (r < held) {
                const float l = lse_of(r);
                if (l != neg_inf_f())  // log2(e) in two parts
                    x = fmaf(-l, kLog2eLow, fmaf(-l, kLog2e, -shift));
            }
            nlse[r] = x;
        }
        fence_async_smem();
        named_sync(kBarW, 256);
    };
    const int page = 1 << a.c.page_shift;
    const int span = min(page, kKeys);  // slots of a page in a tile

    if (warp == S::loader) {
        // ---------------------------------------------------------------- the loading warp
        uint32_t ring = 0;
        const int pieces = kKeys / span;
        while (!dead && next())
            for (int g0 = 0; g0 < a.rows && !dead; g0 += kHeld) {
                int pg_lane = -1;
                for (int t = first; t < last; ++t, ++ring) {
                    const int batch = (t - first) * pieces;
                    if ((batch & 31) == 0) {
                        const int slot = t * kKeys + lane * span;
                        pg_lane = slot < n ? page_of(a.c, a.table, a.max_pages, b, slot) : -2;
                    }
                    const uint32_t st = ring % S::stages;
                    wait(Long{}, kEmpty + st, ((ring / S::stages) & 1) ^ 1);
                    dead = __any_sync(0xFFFFFFFFu, dead);
                    if (dead)
                        break;
                    const int pg = __shfl_sync(0xFFFFFFFFu, pg_lane, (batch & 31) + (lane & 3));
                    const bool mine = lane < pieces && pg >= 0;
                    const uint32_t there = __ballot_sync(0xFFFFFFFFu, mine);
                    const uint32_t bad = __ballot_sync(0xFFFFFFFFu, lane < pieces && pg == -1);
                    if (lane == 0) {
                        bad_pieces[st] = (uint8_t)bad;
                        if (there)
                            mbar_arrive_expect_tx(&bars[kFull + st],
                                                  (uint32_t)__popc(there) * span * (D / 2 + 4));
                        else
                            mbar_arrive(&bars[kFull + st]);
                    }
                    __syncwarp();
                    if (mine) {
                        uint8_t *buf = smem + st * S::stage_bytes;
                        const int in_page = (t * kKeys + lane * span) & (page - 1);
                        const int64_t ph = (int64_t)pg * a.c.heads + h;
                        tma_load_3d(buf + lane * span * (D / 2), &k_map, 0, in_page, (int)ph,
                                    &bars[kFull + st]);
                        bulk_copy_g2s(buf + S::code_bytes + lane * span * 4,
                                      a.c.ka + ph * page + in_page, span * 4, &bars[kFull + st]);
                    }
                    __syncwarp();
                }
            }
        // Nothing may land in this CTA's memory after it has gone.
        for (uint32_t i = 0; i < min(ring, (uint32_t)S::stages); ++i) {
            const uint32_t r = ring - 1 - i;
            if (!mbar_wait_at<100>(bar(kFull + r % S::stages), (r / S::stages) & 1,
                                   dead ? kDrainTries : kWaitTries))
                dead = true;
        }
    } else if (warp == S::issuer) {
        // ---------------------------------------------------------------- the issuing warp
        const uint64_t q_desc = tc::sw128_kmajor_desc(smem + S::q_off);
        uint32_t scores = 0, ring = 0, freed = 0;
        auto wait_warp = [&](int i, uint32_t parity) {
            wait(Now{}, i, parity);
            dead = __any_sync(0xFFFFFFFFu, dead);
        };
        while (!dead && next())
            for (int g0 = 0; g0 < a.rows && !dead; g0 += kHeld) {
                const int held = min(kHeld, a.rows - g0);
                for (int t = first; t < last && !dead; ++t, ++ring) {
                    wait_warp(kKReady, ring & 1);
                    if (dead)
                        break;
                    tc::fence_after_sync();
                    for (int r = 0; r * N < held; ++r, ++scores) {
                        const uint32_t par = scores & 1;
                        if (scores >= 2)
                            wait_warp(kSFree + par, ((scores - 2) >> 1) & 1);
                        if (dead)
                            break;
                        tc::fence_after_sync();
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
                            mma_ts(tmem + S::tS + par * N, tmem + S::tK + 8 * k,
                                   q_desc + r * (S::q_bytes >> 4) +
                                       (k >> 2) * ((N * 128) >> 4) + 2 * (k & 3),
                                   idesc_f16<__half>(128, N, false), k > 0);
                        mma_commit(&bars[kSDone + par]);
                    }
                    mma_commit(&bars[kKFree]);
                    ++freed;
                }
            }
        // Nor may a product read or write what this CTA gives back: the last of them.
        const uint32_t tries = dead ? kDrainTries : kWaitTries;
        if (scores > 0 && !mbar_wait_at<0>(bar(kSDone + ((scores - 1) & 1)), ((scores - 1) >> 1) & 1, tries))
            dead = true;
        if (freed > 0 && !mbar_wait_at<0>(bar(kKFree), (freed - 1) & 1, tries))
            dead = true;
    } else if (warp < 4) {
        // ---------------------------------------------------------------- the unpacking warps
        const int key = tid;
        const uint32_t tK = tmem + ((uint32_t)warp << 21) + S::tK;
        const uint32_t k_row = key * (D / 2) + ((D == 128 ? (key >> 1) & 3 : (key >> 2) & 1) << 4);
        uint32_t ring = 0;  // key tiles so far
        while (next())
            for (int g0 = 0; g0 < a.rows; g0 += kHeld) {
                // the products that read the queries before are done
                if (ring > 0)
                    wait(Short{}, kKFree, (ring - 1) & 1);
                float shift;
                hold_queries(g0, min(kHeld, a.rows - g0), shift);
                for (int t = first; t < last; ++t, ++ring) {
                    const uint32_t st = ring % S::stages;
                    wait(Short{}, kFull + st, (ring / S::stages) & 1);
                    if (ring > 0)  // the products of the tile before have read its keys
                        wait(Short{}, kKFree, (ring - 1) & 1);
                    tc::fence_after_sync();
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        uint32_t y[16];
                        unpack32(lds4(buf0 + st * S::stage_bytes + (k_row ^ (i << 4))), y);
                        tmem_st16(tK + 16 * i, y);
                    }
                    tmem_wait_st();
                    tc::fence_before_sync();
                    __syncwarp();
                    mbar_arrive_if(bar(kKReady), lane == 0);
                    mbar_arrive_if(bar(kEmpty + st), lane == 0);
                }
            }
    } else {
        // ---------------------------------------------------------------- the weighing warps
        const int key = tid - 128;
        const uint32_t tS = tmem + ((uint32_t)(warp & 3) << 21) + S::tS;
        uint32_t ring = 0, scores = 0;
        // What lies behind the lengths is 0; a sequence whose length is out of range is NaN.
        for (int64_t row = blockIdx.x; row < (int64_t)a.B * a.c.heads; row += gridDim.x) {
            const int len = length_of(a, (int)(row / a.c.heads));
            for (int j = max(len, 0) + key; j < a.max_len; j += 128)
                a.out[row * a.max_len + j] = len < 0 ? nan_f() : 0.0f;
        }
        while (next())
            for (int g0 = 0; g0 < a.rows; g0 += kHeld) {
                const int held = min(kHeld, a.rows - g0);
                float shift;
                hold_queries(g0, held, shift);
                const uint64_t shift2 = f2(shift, shift);
                for (int t = first; t < last; ++t, ++ring) {
                    const uint32_t st = ring % S::stages;
                    const int j = t * kKeys + key;
                    const int64_t where = ((int64_t)b * a.c.heads + h) * a.max_len + j;
                    // (a group after the first adds to what this thread wrote)
                    float before = 0.0f;
                    if (j < n && (g0 > 0 || a.in))
                        before = g0 > 0 ? a.out[where] : a.in[where];
                    uint64_t sum2 = 0;
                    float ks = 0.0f, ko = 0.0f;
                    bool bad = false;
                    for (int r = 0; r * N < held; ++r, ++scores) {
                        const uint32_t par = scores & 1;
                        wait(Now{}, kSDone + par, (scores >> 1) & 1);
                        tc::fence_after_sync();
                        if (r == 0) {
                            const uint32_t f = lds1(buf0 + st * S::stage_bytes + S::code_bytes +
                                                    4 * key);
                            ks = bf16_low(f) * a.scale;
                            ko = fmaf(8.0f, bf16_low(f), bf16_high(f)) * a.scale;
                            bad = (bad_pieces[st] >> (key / span)) & 1;
                            __syncwarp();
                            mbar_arrive_if(bar(kEmpty + st), lane == 0);
                        }
                        const uint64_t ks2 = f2(ks, ks), ko2 = f2(ko, ko);
#pragma unroll 1
                        for (int c16 = 0; c16 < N; c16 += 16) {
                            uint32_t s[16];
                            tmem_ld<16>(tS + par * N + c16, s);
                            if (c16 == N - 16) {
                                tc::fence_before_sync();
                                __syncwarp();
                                mbar_arrive_if(bar(kSFree + par), lane == 0);
                            }
#pragma unroll
                            for (int c = 0; c < 16; c += 4) {
                                const float4 sq = lds4f(sum0 + 4 * (r * N + c16 + c));
                                const float4 mq = lds4f(mul0 + 4 * (r * N + c16 + c));
                                const float4 nl = lds4f(lse0 + 4 * (r * N + c16 + c));
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const uint64_t y = fma2(
                                        f2(__uint_as_float(s[c + 2 * e]),
                                           __uint_as_float(s[c + 2 * e + 1])),
                                        ks2, mul2(ko2, e ? f2(sq.z, sq.w) : f2(sq.x, sq.y)));
                                    float y0, y1;
                                    un2(add2(fma2(y, e ? f2(mq.z, mq.w) : f2(mq.x, mq.y), shift2),
                                             e ? f2(nl.z, nl.w) : f2(nl.x, nl.y)),
                                        y0, y1);
                                    sum2 = add2(sum2, f2(ex2_mufu(y0), ex2_mufu(y1)));
                                }
                            }
                        }
                    }
                    float s0, s1;
                    un2(sum2, s0, s1);
                    if (j < n)
                        a.out[where] = bad ? nan_f() : before + (s0 + s1);
                }
            }
    }
    if (dead)
        atomicOr(a.status, kDevStatTimeout);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (warp == S::issuer)
        tc::tmem_dealloc(tmem, S::tmem);
}

// Rows of a row tile: the smallest width that holds a head's rows, 64 beyond that.  (64 sequences
// of 32 heads, 512 keys: 16 rows a head 42 us, in a tile of 32 48, of 64 65; 32 rows 53, of 64 70.)
int tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }

template <typename S, typename T>
cudaError_t run(const WeighArgs &a, const CUtensorMap &k_map, cudaStream_t s)
{
    static PerDevice ready;
    const cudaError_t e = ready.once([] {
        return cudaFuncSetAttribute(weigh_kernel<S, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    S::smem);
    });
    if (e != cudaSuccess)
        return e;
    return launch(weigh_kernel<S, T>, dim3(sm_count() * S::ctas), dim3(S::threads), S::smem, s,
                  true, a, k_map);
}

template <int D, typename T>
cudaError_t run_rows(const WeighArgs &a, const CUtensorMap &k_map, cudaStream_t s)
{
    const int N = tile_rows(a.rows);
    return N == 16   ? run<Shape<D, 16>, T>(a, k_map, s)
           : N == 32 ? run<Shape<D, 32>, T>(a, k_map, s)
                     : run<Shape<D, 64>, T>(a, k_map, s);
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
    a.B = B;
    a.rows = (int)((int64_t)Lq * a.group);
    a.scale = (float)(scale * 1.4426950408889634);
    a.in = weights_in;
    a.out = weights_out;
    a.max_len = max_len;
    CUtensorMap k_map;
    a.status = cache_status_word();
    if (!a.status || !make_cache_maps(a.c, &k_map, nullptr))
        return FDLLM_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf = dtype == FDLLM_BF16;
    const cudaError_t e = a.c.D == 128 ? (bf ? run_rows<128, __nv_bfloat16>(a, k_map, s)
                                             : run_rows<128, __half>(a, k_map, s))
                                       : (bf ? run_rows<64, __nv_bfloat16>(a, k_map, s)
                                             : run_rows<64, __half>(a, k_map, s));
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

}  // extern "C"
