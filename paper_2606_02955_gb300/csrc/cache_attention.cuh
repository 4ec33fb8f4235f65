// cache_attention.cuh -- the kernels of fdllm_cache_attention (cache_attention.cu) and
// fdllm_cache_tree_attention (cache_tree.cu): a block's queries over the 4-bit prefix cache and the
// block's own keys, on the fifth-generation tensor cores.
//
// Mathematics.  With k_j = ko_j + ks_j u_j and v_j = vo_j + vs_j w_j (u_j and w_j the codes less
// a constant, which the offsets ko_j and vo_j make up for), for the rows r of one key/value head
// (queries x heads of the group):
//   s_rj = scale (ks_j (q_r . u_j) + ko_j sum(q_r)),
//   out_r = (sum_j p_rj vs_j w_j + sum_j p_rj vo_j) / sum_j p_rj,   p_rj = e^(s_rj - m_r).
// The tensor cores see the codes themselves, exact in fp16; scales and offsets act on the
// scores and the weights.  Queries enter the first product as fp16 too, times a power of two
// that brings the row's largest to 2^13: exact but for elements below 2^-23 of it.  (One power for
// all rows of a tile took the others' bits where one row's values were 2^20 times theirs, those
// of a padded position for instance.)
//
// Layout.  A tile is 128 keys.  Both products are taken transposed, with the unpacked codes as
// the A operand in tensor memory, so that the codes go from registers straight to the tensor
// core and never back through shared memory:
//   S^T [128 keys x N rows]      = K [keys x D] . Q^T       (a thread holds one key's scores)
//   O^T [128 channels x N rows] += V^T [channels x keys] . P^T
// A key's scale and offset are then scalars of the thread that holds its scores, and V's codes
// are stored channel-major so that a thread unpacks one channel.  P^T is the only operand
// written to shared memory by threads (16-byte stores, rows contiguous).
//
// A row's reference (the running maximum of a softmax) is the largest score of the first 32 keys
// it meets, and moves only when a weight leaves the range that fp16 and fp32 hold (kTopWeight),
// which one vote a tile decides.  Weights are scaled by the cached row's scale before they are
// rounded to fp16; a second reference of the row keeps their largest near 1 whatever the scales
// are.  A weight is held as two numbers of the values' operand type (fp16 for codes, their own
// type for own values): rounded, and what that left times 2^11, as columns of one product with
// sums of their own.  So it keeps 22 bits (16 of bf16), and one far below the largest, a subnormal
// of the first number, keeps its place to 2^-36 of it: a key that outweighs all others at the front
// of a long cache takes nothing from the many small ones behind it.  (With the first number alone
// the results' error was 1.77e-3 for blocks of bf16, of which its rounding is 1.66e-3.)
//
// Warps.  One loads (queries, codes, own keys and values, through one ring of shared-memory
// stages), one issues the products, four unpack, four or eight make weights: an unpacking warp is
// ahead, in the next unit's queries while the weights' warps write a unit's end.
//
// Split.  The tiles of all (sequence, head, row tile) units in order, with a charge of
// kUnitCost tiles for each unit's beginning and end, are cut into equal ranges, one to a CTA
// (the lengths are read on the device); a unit that crosses a CTA's end leaves fp32 partials,
// joined by combine_kernel in tile order.
//
// Bound by the latency of the chain from unpacked keys to given weights and by the instructions
// of the weights (about 350 a warp and tile), then by a unit's beginning and end.  Code that fits the
// instruction cache counts as much as its instructions.  Measured (GPU time, each launch by itself): 64
// sequences of 32 queries and own keys over prefixes of 200 to 1024 keys, 32 heads of 128 channels: 151 us
// (237 MB; the tensor pipe 11 % busy, memory 22 %); 2 sequences of 64 queries of 32 heads over 32000 keys of
// 8: 161 (66 GFLOP); one token of 32 heads over 1021 keys of 8: 13; and 7 for combine_kernel.
#pragma once

#include <cuda_runtime.h>

#include <type_traits>

#include "cache.cuh"
#include "cache_tc.cuh"

namespace fdllm {
namespace {

constexpr int kKeys = 128;                // keys of a tile
constexpr float kFar = -1e30f;            // reference of a row that has seen no key
constexpr float kTopWeight = 16384.0f;    // largest weight (fp16 holds 65504)
constexpr float kTopShift = 90.0f;        // a score this far above its reference may overflow
constexpr float kMaxShift = 120.0f;       // c = 2^-refd stays below 2^120
constexpr int kNever = 0x7FFFFFFF;         // no such key
constexpr float kSumUnit = 1048576.0f;    // sums over values' codes come in units of 2^-20
constexpr float kRest = 2048.0f;          // what a weight's rounding left is held times this

struct AttnArgs {
    CacheView c;
    const int32_t *table;     // [B, max_pages]
    int max_pages;
    const int32_t *lens;      // [B]
    const void *q;            // [B, Lq, Hq, D]
    Strides3 qs;
    int B, Lq, Hq, group;     // group = Hq / heads
    const void *k_new;        // [B, Ln, heads, D]
    const void *v_new;
    Strides3 ks, vs;
    int Ln;
    int mapped;               // own keys and values come by tensor map
    const int32_t *new_lens;  // [B] or null
    int causal;
    const uint32_t *sees;     // [B, Lq, sees_words]: the own keys that a query sees (masked form)
    int sees_words;
    float scale;              // times log2(e)
    void *out;                // [B, Lq, Hq, D]
    float *lse;               // [B, Lq, Hq] or null
    int rows;                 // Lq * group
    int row_tiles;            // ceil(rows / N)
    float *parts;             // [grid][2][N][D] accumulators, at the row's reference
    float *part_refs;         // [grid][2][N][2] (reference, sum)
    int32_t *meta;            // [grid][kMeta]
    uint32_t *status;         // sticky: a bounded wait gave up
};

// meta of a CTA: whether it starts a unit that it does not finish (slot 1) and which, whether
// it continues a unit begun before (slot 0) and whether that ends here.
enum { kOpen = 0, kOpenB, kOpenUnit, kCont, kContEnds, kMeta = 8 };

template <int D_, int N_>
struct Shape {
    static constexpr int D = D_;
    static constexpr int N = N_;                       // rows of a row tile
    // Warpgroups sharing a tile's columns: 16 columns a thread, 32 where the registers are there
    // (32 rows: 164 us, with 32 a thread 180; 64 rows over 32000 keys: 164, with 16 a thread 174).
    static constexpr int C = N <= 32 ? N / 16 : N / 32;
    static constexpr int cols = N / C;                 // columns (rows of the problem) a thread
    static constexpr int w_warps = 4 * C;              // warps that make weights
    static constexpr int w_first = 4;                  // (warps 0 to 3 unpack)
    static constexpr int loader = w_first + w_warps;
    static constexpr int issuer = loader + 1;
    static constexpr int threads = 32 * (loader + 4);  // (two warps of the last group idle)
    static constexpr int ctas = N >= 64 ? 1 : 2;       // CTAs an SM holds
    // Registers of a thread, by warpgroup: what the launch gives every thread is dealt out
    // again, the weights' warps taking what the others leave: spilled registers cost them more than
    // the others (an even share: 224 us for blocks of 32 rows; 40 of 64 for the others: 164, 48: 171).
    static constexpr int regs = 65536 / (ctas * threads) / 8 * 8;
    static constexpr int u_regs = N == 32 ? 40 : 64, l_regs = u_regs;
    static constexpr int w_regs = (regs * (C + 2) - u_regs - l_regs) / C / 8 * 8;
    static_assert(C * w_regs + u_regs + l_regs <= regs * (C + 2) && w_regs >= regs &&
                  u_regs <= regs && l_regs <= regs, "no more than the launch's");
    static constexpr int bufs = ctas == 1 ? 2 : 1;       // of unpacked keys, and of values
    static constexpr int stages = ctas == 1 ? 8 : 4;
    // own keys come 32 to a stage; a block's 32 fill one tile, long prompts whole ones
    static constexpr int own_keys = N >= 64 ? 128 : 32;
    static constexpr int code_bytes = kKeys * D / 2;   // of keys, or of values
    static constexpr int stage_bytes = 2 * code_bytes + 1024;
    // a stage's own keys: 64 channels of 32 rows each, their pieces swizzled by row; then values
    static constexpr int own_v = 64 * D;
    static constexpr int q_bytes = N * D * 2;
    static constexpr int q16_off = stages * stage_bytes;  // queries for codes, in fp16
    static constexpr int qt_off = q16_off + q_bytes;      // queries for own keys, as they are
    static constexpr int p_off = qt_off + q_bytes;
    static constexpr int p_step = 2 * N * 16;  // 8 keys' weights: first numbers, then second ones
    static constexpr int smem = p_off + kKeys / 8 * p_step + 1024;  // and room to align the base
    // tensor memory columns
    // (tO: the sums of the weights' first numbers; tL: of their second)
    static constexpr int tK = 0, tV = 64 * bufs, tS = 128 * bufs, tO = tS + 2 * N, tL = tO + N;
    static constexpr int tmem = tL + N <= 256 ? 256 : 512;
    static_assert(tL + N <= tmem && ctas * tmem <= 512, "tensor memory");
    static_assert(q_bytes <= stage_bytes && own_v + 64 * D <= stage_bytes, "a stage holds them");
    static_assert(stages >= 2 * own_keys / 32, "two own tiles are in flight");
};

// Eight own values of one channel (rows `step` apart in shared memory), as pairs in the operand's
// order; keys from `n` on are 0.  A non-finite value must not meet the zero weights of the rows
// that do not see it: it is taken out, and the first such key returned for the rows that do.
template <typename T>
__device__ __forceinline__ int own_values(const T *v, int step, int n, uint32_t (&y)[4])
{
    constexpr uint32_t kExp = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
    const uint16_t *u = reinterpret_cast<const uint16_t *>(v);
    int bad = 8;
#pragma unroll
    for (int x = 0; x < 4; ++x) {  // and four further on
        uint32_t lo = x < n ? u[x * step] : 0u;
        uint32_t hi = x + 4 < n ? u[(x + 4) * step] : 0u;
        if ((lo & kExp) == kExp)
            bad = min(bad, x), lo = 0;
        if ((hi & kExp) == kExp)
            bad = min(bad, x + 4), hi = 0;
        y[x] = lo | (hi << 16);
    }
    return bad;
}

// Sums in tensor memory times a factor for each column (f) or for all (u).
template <int NC>
__device__ __forceinline__ void scale_sums(uint32_t taddr, const float *f, float u)
{
#pragma unroll 1
    for (int c8 = 0; c8 < NC; c8 += 8) {
        uint32_t s[8];
        tmem_ld<8>(taddr + c8, s);
#pragma unroll
        for (int c = 0; c < 8; ++c)
            s[c] = __float_as_uint(__uint_as_float(s[c]) * (f ? f[c8 + c] : u));
        tmem_st<8>(taddr + c8, s);
    }
    tmem_wait_st();
}

// A unit's beginning and end cost about as much as this many tiles (4 to 8 by the rows; 64 blocks
// of 32 rows: 164 us, with 3 here 165).
constexpr int kUnitCost = 7;

// One sequence's share of the work.
struct Sequence {
    int cached;    // cached keys
    int own;       // own keys
    int ct;        // tiles of cached keys
    int tiles;     // all tiles, at least 1
    bool wrong;    // a length out of range
};

template <int OwnKeys>
__device__ __forceinline__ Sequence sequence_of(const AttnArgs &a, int b)
{
    Sequence s;
    const int n = a.lens[b];
    const int own = a.new_lens ? a.new_lens[b] : a.Ln;
    s.wrong = n < 0 || n > (a.max_pages << a.c.page_shift) || own < 0 || own > a.Ln;
    s.cached = s.wrong ? 0 : n;
    s.own = s.wrong ? 0 : own;
    s.ct = (s.cached + kKeys - 1) / kKeys;
    s.tiles = max(1, s.ct + (s.own + OwnKeys - 1) / OwnKeys);
    return s;
}

// A CTA's walk over its range, segment by segment (a segment: tiles of one unit).
template <int OwnKeys>
struct Walk {
    int64_t at, end;    // places in the whole call
    int64_t base;       // first place of sequence b
    int b;
    Sequence s;
    int unit;           // head * row_tiles + row tile
    int first, last;    // the segment's tiles [first, last) of the unit

    __device__ bool next(const AttnArgs &a, int units)
    {
        while (at < end) {
            while (at >= base + (int64_t)(s.tiles + kUnitCost) * units) {
                base += (int64_t)(s.tiles + kUnitCost) * units;
                s = sequence_of<OwnKeys>(a, ++b);
            }
            const int64_t local = at - base;
            const int length = s.tiles + kUnitCost;
            unit = (int)(local / length);
            const int from = (int)(local - (int64_t)unit * length);
            const int to = (int)min((int64_t)length, from + (end - at));
            at += to - from;
            first = min(from, s.tiles);
            last = min(to, s.tiles);
            if (first < last)
                return true;
        }
        return false;
    }
};

// What a segment's warps need to know of it, left in shared memory by the loading warp.
struct Segment {
    int b, unit, h, r0, rows;  // sequence; head * row_tiles + row tile; head; rows r0 ...
    int first, last;           // tiles of the unit that hold keys, [first, last)
    int ct, cached, own;
    int starts, ends;          // the unit's first tile, its last
    int wrong;
    int done;                  // no segment: the walk is over
};

// Whether query `qi` sees a non-finite value of channel d among the segment's own keys (where some
// query may: the values are read again).
template <typename T>
__device__ __noinline__ bool meets_bad(const AttnArgs &a, const Segment &g, int qi, int d, int own_keys)
{
    constexpr uint32_t kExp = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;
    const uint32_t *sees = a.sees + ((int64_t)g.b * a.Lq + qi) * a.sees_words;
    const uint16_t *v = static_cast<const uint16_t *>(a.v_new) + g.b * a.vs.batch + g.h * a.vs.head + d;
    const int to = min(g.own, (g.last - g.ct) * own_keys);
    for (int j = max(g.first - g.ct, 0) * own_keys; j < to; ++j)
        if ((sees[j >> 5] >> (j & 31)) & 1u && (v[j * a.vs.token] & kExp) == kExp)
            return true;
    return false;
}

// Lane i's bit k becomes lane k's bit i.
__device__ __forceinline__ uint32_t transpose_bits(uint32_t x)
{
    const int lane = threadIdx.x & 31;
    uint32_t keep = 0x0000FFFFu;
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) {
        const uint32_t y = __shfl_xor_sync(0xFFFFFFFFu, x, m);
        x = lane & m ? (x & ~keep) | ((y & ~keep) >> m) : (x & keep) | ((y & keep) << m);
        keep ^= keep << (m >> 1);
    }
    return x;
}

// kMasked: a query sees the own keys whose bits are set in its row of a.sees (a tree's ancestors);
// else all of them, or with a.causal those up to itself.
template <typename S, typename T, bool kMasked>
__global__ void __launch_bounds__(S::threads, S::ctas)
    attention_kernel(const __grid_constant__ AttnArgs a,
                     const __grid_constant__ CUtensorMap k_map,
                     const __grid_constant__ CUtensorMap v_map,
                     const __grid_constant__ CUtensorMap kn_map,
                     const __grid_constant__ CUtensorMap vn_map)
{
    constexpr int D = S::D, N = S::N, kCols = S::cols, kOwnKeys = S::own_keys;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    // Memory barriers: the ring's stages full and empty; of a segment, by its parity, published
    // and done with; of a tile, by its parity, scores and sums done, keys and values
    // unpacked; weights given.  Every wait follows its barrier phase by phase (one that was two
    // phases ahead would take the phase before last for its own).
    enum {
        kFull = 0, kEmpty = kFull + S::stages, kSegFull = kEmpty + S::stages, kSegEmpty = kSegFull + 2,
        kSDone = kSegEmpty + 2, kODone = kSDone + 2, kKReady = kODone + 2, kVReady = kKReady + 2,
        kPReady = kVReady + 2, kBars
    };
    enum { kBarU = 1, kBarW };  // CTA barriers: the unpacking warps, each warpgroup of weights
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ uint32_t tmem_base;
    __shared__ int64_t scan[S::threads / 32];
    __shared__ int64_t find_base;
    __shared__ int find_b;
    // of a segment, by its parity: what it is, whether it met a page out of range, a score's
    // unit, the first own key with a non-finite value (by channel)
    __shared__ Segment segs[2];
    __shared__ int bad_page[2], any_bad[2];
    __shared__ int first_bad[2][D];
    // per row: the reference (negated), 2^-refd, the queries' sums (by the segment's
    // parity); -inf, the references of absent keys; the scaled weights' reference less the row's
    // (apart, so that references of 2^24 and more leave it its bits); factors;
    // the queries' units (by the segment's parity)
    enum { kNref = 0, kCmul = N, kSumq = 2 * N, kNone = 4 * N, kRefd = 5 * N, kFl = 6 * N,
           kFo = 7 * N, kRedo = 8 * N, kMulq = 9 * N, kRowFloats = 11 * N };
    __shared__ __align__(16) float rowf[kRowFloats];
    float *const nref = rowf + kNref, *const cmul = rowf + kCmul, *const refd = rowf + kRefd;
    float *const fl = rowf + kFl, *const fo = rowf + kFo, *const redo = rowf + kRedo;
    // by the segment's parity: where a row's results go (in rows of D), their factors (of the
    // sums, and added), and sums of each warp's keys
    __shared__ int64_t row_at[2][N];
    __shared__ float2 fin[2][N];
    __shared__ float wred[2][S::w_warps][2][kCols];

    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < kBars; ++i) {
            const int n = i >= kEmpty && i < kSegFull     ? 4 + S::w_warps
                          : i >= kSegEmpty && i < kSDone ? 4 + S::w_warps + 1
                          : i >= kKReady && i < kPReady  ? 4
                          : i == kPReady                 ? S::w_warps
                                                         : 1;
            mbar_init(&bars[i], n);
        }
        fence_mbar_init();
    }
    if (tid < N)
        rowf[kNone + tid] = neg_inf_f();
    if (warp == S::issuer)
        tc::tmem_alloc(&tmem_base, S::tmem);
    if (warp == S::loader && lane == 0) {
        tc::prefetch_tensormap(&k_map);
        tc::prefetch_tensormap(&v_map);
        if (a.mapped) {
            tc::prefetch_tensormap(&kn_map);
            tc::prefetch_tensormap(&vn_map);
        }
    }
    pdl_wait();

    // The call's places, and the sequence in which this CTA's range begins: every thread sums a
    // run of sequences, a scan over the CTA gives the runs' places.
    const int units = a.c.heads * a.row_tiles;
    Walk<kOwnKeys> w;
    {
        const int run = (a.B + S::threads - 1) / S::threads;
        const int b0 = min(a.B, tid * run), b1 = min(a.B, b0 + run);
        int64_t mine = 0;
        for (int b = b0; b < b1; ++b)
            mine += sequence_of<kOwnKeys>(a, b).tiles + kUnitCost;
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
        total *= units;
        const int64_t p0 = (before + upto - mine) * units;
        w.at = total * blockIdx.x / gridDim.x;
        w.end = total * (blockIdx.x + 1) / gridDim.x;
        if (b0 < b1 && w.at >= p0 && w.at < p0 + mine * units) {
            find_base = p0;
            find_b = b0;
        }
    }
    int32_t *meta = a.meta + (int64_t)blockIdx.x * kMeta;
    if (tid < kMeta)
        meta[tid] = 0;
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, tmem_base, 0);
    pdl_launch_dependents();

    // Addresses of the barriers and of the dynamic memory, kept rather than rebuilt.
    uint32_t bar0 = smem_addr(bars), buf0 = smem_addr(smem), row0 = smem_addr(rowf);
    asm volatile("" : "+r"(bar0), "+r"(buf0), "+r"(row0));
    auto bar = [&](int i) { return bar0 + 8u * i; };
    // A wait gave up: no further wait.  The loading and the issuing warp stop (the former says that
    // there are no more segments) and wait, with a limit, for what they have in flight; the others
    // finish their segment, whose places are still good, and leave together, by a vote, before the
    // next, which may never have been published.
    bool dead = false;
    auto wait = [&](int i, uint32_t parity) {
        if (!dead && !mbar_wait_at<0>(bar(i), parity))
            dead = true;
    };
    auto wait_u = [&](int i, uint32_t parity) {
        if (!dead && !mbar_wait_at<20>(bar(i), parity))
            dead = true;
    };
    // the same for a whole warp that waits most of its time
    auto wait_warp = [&](auto sleep, int i, uint32_t parity) {
        if (!dead && !mbar_wait_at<decltype(sleep)::value>(bar(i), parity))
            dead = true;
        dead = __any_sync(0xFFFFFFFFu, dead);
    };
    using Long = std::integral_constant<int, 100>;
    using Now = std::integral_constant<int, 0>;

    if (warp >= S::loader)
        reg_dec<S::l_regs>();
    if (warp == S::loader) {
        // ---------------------------------------------------------------- the loading warp
        if (w.at < w.end) {
            w.b = find_b;
            w.base = find_base;
            w.s = sequence_of<kOwnKeys>(a, w.b);
        }
        uint32_t ring = 0;  // stages filled so far: stage ring % stages, phase ring / stages
        const int page = 1 << a.c.page_shift;
        const int span = min(page, kKeys);  // slots of a page in a tile
        const int pieces = kKeys / span;
        for (uint32_t seg = 0;; ++seg) {
            const uint32_t sb = seg & 1;
            bool more = w.next(a, units);
            wait_warp(Long{}, kSegEmpty + (sb), ((seg >> 1) & 1) ^ 1);
            more = more && !dead;  // (64 blocks with a `break` here: 180 us, as compiled, not 161)
            const int h = more ? w.unit / a.row_tiles : 0;
            const int r0 = more ? (w.unit - h * a.row_tiles) * N : 0;
            const int rows = min(N, a.rows - r0);
            int own_tiles = more ? (w.s.own + kOwnKeys - 1) / kOwnKeys : 0;
            if (a.causal)  // own keys that the last row sees
                own_tiles = min(own_tiles, (r0 + rows - 1) / a.group / kOwnKeys + 1);
            const int last = more ? min(w.last, w.s.ct + own_tiles) : 0;
            if (lane == 0) {
                Segment &g = segs[sb];
                g.done = !more;
                if (more) {
                    g.b = w.b, g.unit = w.unit, g.h = h, g.r0 = r0, g.rows = rows;
                    g.first = w.first, g.last = last;
                    g.ct = w.s.ct, g.cached = w.s.cached, g.own = w.s.own;
                    g.starts = w.first == 0, g.ends = w.last == w.s.tiles;
                    g.wrong = w.s.wrong;
                    bad_page[sb] = 0;
                }
            }
            if (more) {
                const bool starts = w.first == 0, whole = starts && w.last == w.s.tiles;
                for (int n = lane; n < rows; n += 32) {
                    const int qi = (r0 + n) / a.group, j = (r0 + n) - qi * a.group;
                    row_at[sb][n] = whole ? ((int64_t)w.b * a.Lq + qi) * a.Hq + h * a.group + j
                                          : ((int64_t)blockIdx.x * 2 + starts) * N + n;
                }
            }
            __syncwarp();
            if (lane == 0)
                mbar_arrive(&bars[kSegFull + (sb)]);
            __syncwarp();
            if (!more)
                break;
            if (w.first >= last)
                continue;
            // The queries' rows.
            {
                const uint32_t st = ring % S::stages;
                wait_warp(Long{}, kEmpty + (st), ((ring / S::stages) & 1) ^ 1);
                if (dead)
                    break;
                uint8_t *buf = smem + st * S::stage_bytes;
                if (lane == 0)
                    mbar_arrive_expect_tx(&bars[kFull + st], (uint32_t)rows * D * 2);
                __syncwarp();
                for (int n = lane; n < rows; n += 32) {
                    const int qi = (r0 + n) / a.group, g = (r0 + n) - qi * a.group;
                    bulk_copy_g2s(buf + n * (D * 2),
                                  static_cast<const T *>(a.q) + w.b * a.qs.batch +
                                      qi * a.qs.token + (int64_t)(h * a.group + g) * a.qs.head,
                                  D * 2, &bars[kFull + st]);
                }
                ++ring;
            }
            // Cached tiles; a lane looks up one page of the next 32.
            const int cached_end = min(last, w.s.ct);
            int pg_lane = -1;
            for (int t = w.first; t < cached_end; ++t, ++ring) {
                const int batch = (t - w.first) * pieces;  // pieces since the segment began
                if ((batch & 31) == 0) {
                    const int slot = t * kKeys + lane * span;
                    pg_lane = slot < w.s.cached
                                  ? page_of(a.c, a.table, a.max_pages, w.b, slot)
                                  : -2;
                }
                const uint32_t st = ring % S::stages;
                wait_warp(Long{}, kEmpty + (st), ((ring / S::stages) & 1) ^ 1);
                if (dead)
                    break;
                uint8_t *buf = smem + st * S::stage_bytes;
                // lane i < pieces copies piece i
                const int pg = __shfl_sync(0xFFFFFFFFu, pg_lane, (batch & 31) + (lane & 3));
                const bool mine = lane < pieces && pg >= 0;
                const uint32_t there = __ballot_sync(0xFFFFFFFFu, mine);
                const bool bad = __any_sync(0xFFFFFFFFu, lane < pieces && pg == -1);
                if (lane == 0) {
                    if (bad)
                        bad_page[sb] = 1;
                    if (there)
                        mbar_arrive_expect_tx(&bars[kFull + st],
                                              (uint32_t)__popc(there) * span * (D + 8));
                    else
                        mbar_arrive(&bars[kFull + (st)]);
                }
                __syncwarp();
                if (mine) {
                    const int i = lane;
                    const int in_page = (t * kKeys + i * span) & (page - 1);
                    const int64_t ph = (int64_t)pg * a.c.heads + h;
                    tma_load_3d(buf + i * span * (D / 2), &k_map, 0, in_page, (int)ph,
                                &bars[kFull + st]);
                    tma_load_3d(buf + S::code_bytes + i * (span / 2) * D, &v_map, in_page / 2, 0,
                                (int)ph, &bars[kFull + st]);
                    uint8_t *aff = buf + 2 * S::code_bytes + i * span * 4;
                    bulk_copy_g2s(aff, a.c.ka + ph * page + in_page, span * 4, &bars[kFull + st]);
                    bulk_copy_g2s(aff + 512, a.c.va + ph * page + in_page, span * 4, &bars[kFull + st]);
                }
                __syncwarp();
            }
            // Own tiles, 32 keys and values to a stage.
            for (int t = max(w.first, w.s.ct); t < last && !dead; ++t) {
                const int j1 = min(w.s.own, (t - w.s.ct + 1) * kOwnKeys);
                for (int j0 = (t - w.s.ct) * kOwnKeys; j0 < j1; j0 += 32, ++ring) {
                    const uint32_t st = ring % S::stages;
                    wait_warp(Long{}, kEmpty + (st), ((ring / S::stages) & 1) ^ 1);
                    uint8_t *buf = smem + st * S::stage_bytes;
                    const int n = min(32, j1 - j0);
                    if (dead)
                        break;
                    if (a.mapped) {
                        if (lane == 0) {
                            mbar_arrive_expect_tx(&bars[kFull + st], 32 * D * 4);
#pragma unroll
                            for (int i = 0; i < D / 64; ++i)
                                tma_load_4d(buf + i * 4096, &kn_map, 64 * i, h, j0, w.b,
                                            &bars[kFull + st]);
                            tma_load_4d(buf + S::own_v, &vn_map, 0, h, j0, w.b, &bars[kFull + st]);
                        }
                    } else {  // rows that repeat: as a map would lay them out
                        if (lane == 0)
                            mbar_arrive_expect_tx(&bars[kFull + st], (uint32_t)n * D * 4);
                        __syncwarp();
                        if (lane < n) {
                            const T *k = static_cast<const T *>(a.k_new) + w.b * a.ks.batch +
                                         (int64_t)(j0 + lane) * a.ks.token + (int64_t)h * a.ks.head;
#pragma unroll 1
                            for (int i = 0; i < D / 8; ++i)
                                bulk_copy_g2s(buf + (i >> 3) * 4096 + lane * 128 +
                                                  (((i & 7) ^ (lane & 7)) << 4),
                                              k + 8 * i, 16, &bars[kFull + st]);
                            bulk_copy_g2s(buf + S::own_v + lane * (D * 2),
                                          static_cast<const T *>(a.v_new) + w.b * a.vs.batch +
                                              (int64_t)(j0 + lane) * a.vs.token +
                                              (int64_t)h * a.vs.head,
                                          D * 2, &bars[kFull + st]);
                        }
                    }
                    __syncwarp();
                }
            }
        }
        // Nothing may land in this CTA's memory after it has gone: the last copies of every
        // stage (at most one round each) are waited for, with a limit.
        __syncwarp();
        for (uint32_t i = 0; i < min(ring, (uint32_t)S::stages); ++i) {
            const uint32_t r = ring - 1 - i;
            if (!mbar_wait_at<100>(bar(kFull + r % S::stages), (r / S::stages) & 1,
                                   dead ? kDrainTries : kWaitTries))
                dead = true;
        }
    } else if (warp == S::issuer) {
        // ---------------------------------------------------------------- the issuing warp
        // S of a tile before the sums of the tile before it, so that the tensor core works on
        // scores while the others make weights.
        const uint64_t q16_desc = tc::sw128_kmajor_desc(smem + S::q16_off);
        const uint64_t qt_desc = tc::sw128_kmajor_desc(smem + S::qt_off);
        const uint64_t p_desc = mn_desc(smem + S::p_off, 128, S::p_step);
        uint32_t scores = 0, sums = 0;  // tiles issued so far
        for (uint32_t seg = 0;; ++seg) {
            const uint32_t sb = seg & 1;
            wait_warp(Now{}, kSegFull + (sb), (seg >> 1) & 1);
            if (dead)
                break;
            const int done = segs[sb].done, first = segs[sb].first, last = segs[sb].last;
            const int ct = segs[sb].ct, own_total = segs[sb].own;
            __syncwarp();
            if (lane == 0)
                mbar_arrive(&bars[kSegEmpty + (sb)]);
            if (done)
                break;
            for (int t = first; t <= last; ++t) {
                if (t < last) {
                    const uint32_t par = scores & 1;
                    wait_warp(Now{}, kKReady + par, (scores >> 1) & 1);
                    if (dead)
                        break;
                    tc::fence_after_sync();
                    const uint64_t q_desc = t < ct ? q16_desc : qt_desc;
                    const uint32_t idesc =
                        t < ct ? idesc_f16<__half>(128, N, false) : idesc_f16<T>(128, N, false);
                    const uint32_t tK = tmem + S::tK + (S::bufs > 1 ? par * 64 : 0);
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        mma_ts(tmem + S::tS + par * N, tK + 8 * k,
                               q_desc + (k >> 2) * ((N * 128) >> 4) + 2 * (k & 3), idesc, k > 0);
                    mma_commit(&bars[kSDone + par]);
                    ++scores;
                }
                if (t > first) {
                    const uint32_t par = sums & 1;
                    wait_warp(Now{}, kVReady + par, (sums >> 1) & 1);
                    wait_warp(Now{}, kPReady, sums & 1);
                    if (dead)
                        break;
                    tc::fence_after_sync();
                    const uint32_t tV = tmem + S::tV + (S::bufs > 1 ? par * 64 : 0);
                    const uint32_t more = t - 1 > first;
                    if (t - 1 < ct) {
                        constexpr uint32_t idesc = idesc_f16<__half>(128, 2 * N, true);
#pragma unroll
                        for (int k = 0; k < kKeys / 16; ++k)
                            mma_ts(tmem + S::tO, tV + 8 * k, p_desc + k * ((2 * S::p_step) >> 4),
                                   idesc, k > 0 ? 1u : more);
                    } else {
                        constexpr uint32_t idesc = idesc_f16<T>(128, 2 * N, true);
                        const int keys = min(kOwnKeys, own_total - (t - 1 - ct) * kOwnKeys);
                        const int steps = (keys + 31) / 32 * 2;
                        for (int k = 0; k < steps; ++k)
                            mma_ts(tmem + S::tO, tV + 8 * k, p_desc + k * ((2 * S::p_step) >> 4),
                                   idesc, k > 0 ? 1u : more);
                    }
                    mma_commit(&bars[kODone + par]);
                    ++sums;
                }
            }
            if (dead)
                break;
        }
        // Nor may a product read or write what this CTA gives back: the last of either kind.
        const uint32_t tries = dead ? kDrainTries : kWaitTries;
        if (scores > 0 && !mbar_wait_at<0>(bar(kSDone + ((scores - 1) & 1)), ((scores - 1) >> 1) & 1, tries))
            dead = true;
        if (sums > 0 && !mbar_wait_at<0>(bar(kODone + ((sums - 1) & 1)), ((sums - 1) >> 1) & 1, tries))
            dead = true;
    } else if (warp > S::issuer) {
        // nothing to do
    } else if (warp < S::w_first) {
        reg_dec<S::u_regs>();
        // ---------------------------------------------------------------- the unpacking warps
        // Queries, keys and values into the tensor core's operands; a thread is a key of K and
        // a channel of V^T.
        const int key = tid;
        const uint32_t lanes = tmem + ((uint32_t)warp << 21);
        uint32_t ring = 0, tile = 0;  // stages used, tiles unpacked so far
        auto arrive = [&](int i, uint32_t n) {
            __syncwarp();
            mbar_arrive_if(bar(i), lane == 0, n);
        };
        // Where this thread's row of codes lies in a stage: 16-byte pieces, swizzled as the
        // tensor maps say.
        const uint32_t k_row = key * (D / 2) + ((D == 128 ? (key >> 1) & 3 : (key >> 2) & 1) << 4);
        uint32_t v_piece[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = key;
            v_piece[i] = S::code_bytes;
            if (a.c.page_shift == 5)
                v_piece[i] += i * (16 * D) + d * 16;
            else if (a.c.page_shift == 6)
                v_piece[i] += (i >> 1) * (32 * D) + d * 32 + (((i & 1) ^ ((d >> 2) & 1)) << 4);
            else
                v_piece[i] += d * 64 + ((i ^ ((d >> 1) & 3)) << 4);
        }
        // Stages that only these warps read are given back for all.
        constexpr uint32_t kForAll = 1 + S::C;
        for (uint32_t seg = 0;; ++seg) {
            const uint32_t sb = seg & 1;
            wait_u(kSegFull + (sb), (seg >> 1) & 1);
            if (tid < D)
                first_bad[sb][tid] = kNever;
            if (tid == 0)
                any_bad[sb] = 0;
            const Segment &g = segs[sb];
            if (named_sync_or(kBarU, 128, dead || g.done))
                break;
            const int first = g.first, last = g.last, ct = g.ct, own = g.own;
            if (first < last) {
                // ---- the queries: their sums, and both operands (K-major, 128-byte swizzle)
                const uint32_t st = ring % S::stages;
                wait_u(kFull + (st), (ring / S::stages) & 1);
                const uint8_t *raw = smem + st * S::stage_bytes;
                constexpr int kMine = N * (D / 8) / 128;
                // the operands' last readers are done: the scores of the tile before
                if (tile > 0)
                    wait_u(kSDone + ((tile - 1) & 1), ((tile - 1) >> 1) & 1);
#pragma unroll 1
                for (int m = 0; m < kMine; ++m) {
                    const int i = tid + m * 128, n = i / (D / 8), c8 = i % (D / 8);
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (n < g.rows)
                        x = *reinterpret_cast<const uint4 *>(raw + 16 * i);
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
                        rowf[kSumq + sb * N + n] = sum * unit;
                        rowf[kMulq + sb * N + n] = power_of_two(e);
                    }
                    const int at = (c8 >> 3) * (N * 128) + n * 128 + (((c8 & 7) ^ (n & 7)) << 4);
                    *reinterpret_cast<uint4 *>(smem + S::q16_off + at) = code_queries<T>(x, unit);
                    if (last > ct)
                        *reinterpret_cast<uint4 *>(smem + S::qt_off + at) = interleave8(x);
                }
                fence_async_smem();  // for the first tile's product
                arrive(kEmpty + st, kForAll);
                ++ring;
            }
            // A tile's values come with its keys.  (The next tile's keys first: 164 us for 64 blocks
            // of 32 rows, not 156; 970 for prompts of 8 x 1021, not 829; 161, not 163, for 64 rows over
            // 32000 keys.)
            for (int t = first; t < last; ++t, ++tile) {
                const uint32_t par = tile & 1;
                const bool cached = t < ct;
                const int keys = cached ? kKeys : min(kOwnKeys, own - (t - ct) * kOwnKeys);
                const int used = cached ? 1 : (keys + 31) / 32;
                // ---- keys; their place is free when the scores of `bufs` tiles before are done
                const uint32_t tK = lanes + S::tK + (S::bufs > 1 ? par * 64 : 0);
                if (tile >= S::bufs)
                    wait_u(kSDone + ((tile - S::bufs) & 1), ((tile - S::bufs) >> 1) & 1);
                if (cached) {
                    const uint32_t s1 = ring % S::stages;
                    wait_u(kFull + (s1), (ring / S::stages) & 1);
                    tc::fence_after_sync();
                    const uint32_t row = buf0 + s1 * S::stage_bytes;
#pragma unroll
                    for (int v = 0; v < D / 32; ++v) {
                        uint32_t y[16];
                        unpack32(lds4(row + (k_row ^ (v << 4))), y);
                        tmem_st16(tK + 16 * v, y);
                    }
                } else if (32 * warp < keys) {
                    const uint32_t r = ring + warp, s1 = r % S::stages;
                    wait_u(kFull + (s1), (r / S::stages) & 1);
                    tc::fence_after_sync();
                    const uint8_t *row = smem + s1 * S::stage_bytes + lane * 128;
#pragma unroll 1
                    for (int v = 0; v < D / 8; ++v) {
                        uint4 x = make_uint4(0, 0, 0, 0);
                        if (key < keys)
                            x = interleave8(*reinterpret_cast<const uint4 *>(
                                row + (v >> 3) * 4096 + (((v & 7) ^ (lane & 7)) << 4)));
                        const uint32_t y[4] = {x.x, x.y, x.z, x.w};
                        tmem_st<4>(tK + 4 * v, y);
                    }
                }
                tmem_wait_st();
                tc::fence_before_sync();
                arrive(kKReady + par, 1);
                // ---- values; their place is free when the sums of `bufs` tiles before are done
                const uint32_t tV = lanes + S::tV + (S::bufs > 1 ? par * 64 : 0);
                if (tile >= S::bufs)
                    wait_u(kODone + ((tile - S::bufs) & 1), ((tile - S::bufs) >> 1) & 1);
                tc::fence_after_sync();
                const int d = key;
                if (cached) {
                    const uint32_t at = buf0 + (ring % S::stages) * S::stage_bytes;
                    if (D == 128 || d < D)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {  // 32 slots
                            uint32_t y[16];
                            unpack32_values(lds4(at + v_piece[v]), y);
                            tmem_st16(tV + 16 * v, y);
                        }
                    tmem_wait_st();
                    tc::fence_before_sync();
                    arrive(kVReady + par, 1);
                    arrive(kEmpty + (ring % S::stages), 1);
                } else {
#pragma unroll 1
                    for (int v = 0; v < used; ++v) {
                        const uint32_t r = ring + v, s1 = r % S::stages;
                        wait_u(kFull + (s1), (r / S::stages) & 1);
                        if (D == 128 || d < D)
#pragma unroll 1
                            for (int j = 0; j < 32; j += 8) {
                                uint32_t y[4];
                                const int bad = own_values<T>(
                                    reinterpret_cast<const T *>(smem + s1 * S::stage_bytes +
                                                                S::own_v) + j * D + d,
                                    D, keys - 32 * v - j, y);
                                if (bad < 8) {
                                    first_bad[sb][d] = min(
                                        first_bad[sb][d], (t - ct) * kOwnKeys + 32 * v + j + bad);
                                    any_bad[sb] = 1;
                                }
                                tmem_st<4>(tV + 16 * v + j / 2, y);
                            }
                    }
                    tmem_wait_st();
                    tc::fence_before_sync();
                    arrive(kVReady + par, 1);
                    for (int v = 0; v < used; ++v)
                        arrive(kEmpty + ((ring + v) % S::stages), kForAll);
                }
                ring += used;
            }
            arrive(kSegEmpty + (sb), 1);
        }
    } else {
        reg_inc<S::w_regs>();
        // ---------------------------------------------------------------- the weights
        // A thread holds one key's scores of its columns.  Each warpgroup has columns of its
        // own, and waits for no other.
        const int wt = tid - 32 * S::w_first, ww = warp - S::w_first;  // thread, warp among these
        const int wg = ww >> 2, quarter = ww & 3, key = wt & 127;
        const int col0 = wg * kCols;  // this thread's columns
        const uint32_t lanes = tmem + ((uint32_t)quarter << 21);
        // where this thread's weights go: 16 bytes (8 rows of its key) a column group
        const int kappa = (key & ~7) | ((key & 3) << 1) | ((key >> 2) & 1);
        const uint32_t p_at = buf0 + S::p_off + (kappa >> 3) * S::p_step + (col0 >> 3) * 128 +
                              (kappa & 7) * 16;
        const uint32_t cols_at = row0 + 4 * col0;
        uint32_t ring = 0;    // stages used so far
        uint32_t seen = 0;    // tiles whose weights were given
        uint32_t summed = 0;  // tiles whose sums were waited for
        auto sync = [&] { named_sync(kBarW + wg, 128); };

        for (uint32_t seg = 0;; ++seg) {
            const uint32_t sb = seg & 1;
            wait(kSegFull + (sb), (seg >> 1) & 1);
            const Segment &g = segs[sb];
            if (named_sync_or(kBarW + wg, 128, dead || g.done))
                break;
            const int begin = g.first;
            const bool some = begin < g.last;
            ring += some ? 1 : 0;  // the queries'
            uint64_t l2[kCols / 2], pm2[kCols / 2];
#pragma unroll
            for (int j = 0; j < kCols / 2; ++j)
                l2[j] = pm2[j] = 0;

            // Tiles [from, to) of the unit, all of them cached or all of them own.
            auto tiles = [&](auto own_tag, int from, int to) {
                constexpr bool kOwn = decltype(own_tag)::value;
                using W = std::conditional_t<kOwn, T, __half>;  // weights and values
                const int end = kOwn ? g.own : g.cached;
                const int base = kOwn ? g.ct : 0;
                constexpr int step = kOwn ? kOwnKeys : kKeys;
#pragma unroll 1
                for (int t = from; t < to; ++t) {
                    const int keys = min(step, end - (t - base) * step);
                    const uint32_t st = ring % S::stages;
                    const uint32_t tS = lanes + S::tS + (seen & 1) * N + col0;
                    [[maybe_unused]] uint32_t my_sees = 0;  // lane c: column c's bits of this warp's keys
                    if constexpr (kOwn && kMasked) {
                        const int word = (t - base) * (step / 32) + quarter, n = g.r0 + col0 + lane;
                        if (lane < kCols && n < a.rows && 32 * quarter < keys)
                            my_sees = __ldg(a.sees + ((int64_t)g.b * a.Lq + n / a.group) * a.sees_words + word);
                    }
                    wait(kSDone + (seen & 1), (seen >> 1) & 1);
                    tc::fence_after_sync();
                    // this thread's key: scale and offset, for scores and weights
                    const int j = (t - base) * step + key;
                    const bool valid = key < keys;
                    float ks = a.scale, ko = 0.0f, vs = 1.0f, vo = 0.0f;
                    if constexpr (!kOwn) {
                        const uint32_t f = buf0 + st * S::stage_bytes + 2 * S::code_bytes + 4 * key;
                        const uint32_t fk = lds1(f), fv = lds1(f + 4 * kKeys);
                        ks = bf16_low(fk) * a.scale;
                        ko = fmaf(8.0f, bf16_low(fk), bf16_high(fk)) * a.scale;
                        vs = bf16_low(fv);
                        vo = fmaf(key & 1 ? 15.0f : 0.0f, vs, bf16_high(fv));
                        if (!valid)
                            ks = ko = vs = vo = 0.0f;
                    }
                    // values' codes of odd slots are 16 times as large: their weights are not
                    const float vw = kOwn || (key & 1) ? vs : 16.0f * vs;
                    // a score of this key, as the weights' are computed (times a power of two)
                    auto score = [&](uint32_t s, int c) {
                        if constexpr (kOwn)
                            return __fmul_rn(__uint_as_float(s), ks);
                        else
                            return fmaf(__uint_as_float(s), ks, ko * rowf[kSumq + sb * N + col0 + c]) *
                                   rowf[kMulq + sb * N + col0 + c];
                    };
                    // the rows of this thread that see its key: those from first_col on
                    [[maybe_unused]] const int first_col =
                        !valid || (kOwn && a.causal && j >= a.Lq) ? kCols
                        : kOwn && a.causal                        ? j * a.group - (g.r0 + col0)
                                                                  : 0;
                    [[maybe_unused]] uint32_t sees = 0;  // or a bit for each
                    if constexpr (kOwn && kMasked) {
                        sees = transpose_bits(my_sees);
                        if (!valid)
                            sees = 0;
                    }
                    auto seen_by = [&](int c) {
                        if constexpr (kOwn && kMasked)
                            return ((sees >> c) & 1u) != 0;
                        else
                            return c >= first_col;
                    };
                    if (__builtin_expect(t == begin, 0)) {
                        // ---- the references: the largest score of the tile's first 32 keys
                        // that the row sees, with the largest scale of their values
                        if (quarter == 0) {
                            const float big = __uint_as_float(
                                __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(fmaxf(vs, 0.0f))));
                            const float small = __uint_as_float(__reduce_min_sync(
                                0xFFFFFFFFu, vs > 0.0f ? __float_as_uint(vs) : 0x7F800000u));
                            // scales within a factor of 2^8: the largest stands for all
                            const bool alike = !(big > 256.0f * small);
                            const float lv = vs > 0.0f ? log2f(vs) : neg_inf_f();
#pragma unroll 1
                            for (int c8 = 0; c8 < kCols; c8 += 8) {
                                float x[8];
                                // lane c: column c's largest score, or score over `ref` and more
                                auto largest = [&](bool over_ref, float ref, float more) {
                                    uint32_t s[8];
                                    tmem_ld<8>(tS + c8, s);
#pragma unroll
                                    for (int c = 0; c < 8; ++c) {
                                        float y = score(s[c], c8 + c);
                                        if (over_ref)
                                            y = (y - __shfl_sync(0xFFFFFFFFu, ref, c)) + more;
                                        x[c] = seen_by(c8 + c) ? y : neg_inf_f();
                                    }
                                    warp_columns<8>(x, [](float u, float v) { return fmaxf(u, v); });
                                    return x[0] == neg_inf_f()    ? kFar
                                           : fabsf(x[0]) < 1e30f ? x[0]
                                                                 : 0.0f;
                                };
                                const float ref = largest(false, 0.0f, 0.0f);
                                float z = -kMaxShift;
                                if (!alike)
                                    z = fmaxf(z, largest(true, ref, lv));
                                else if (big > 0.0f)
                                    z = fmaxf(z, log2f(big));
                                if (lane < 8) {
                                    const int n = col0 + c8 + lane;
                                    nref[n] = -ref;
                                    refd[n] = z;
                                    cmul[n] = ref == kFar ? 1.0f : exp2f(-z);
                                }
                            }
                        }
                        sync();
                    }
                    uint32_t ph[kCols / 2], pl[kCols / 2];
                    // Weights of this thread's columns, and their sums.  The second time (after
                    // the references moved) only the rows of `redo` are summed again.
                    auto weights = [&](auto again) -> float {
                        constexpr bool kAgain = decltype(again)::value;
                        const uint32_t nr_at = valid ? cols_at + 4 * kNref : cols_at + 4 * kNone;
                        [[maybe_unused]] const uint32_t sq_at = cols_at + 4 * (kSumq + sb * N);
                        [[maybe_unused]] const uint32_t mq_at = cols_at + 4 * (kMulq + sb * N);
                        const uint64_t ks2 = f2(ks, ks), ko2 = f2(ko, ko);
                        const uint64_t vw2 = f2(vw, vw), vo2 = f2(vo, vo);
                        float top = 0.0f;
#pragma unroll
                        for (int c8 = 0; c8 < kCols; c8 += 8) {
                            uint32_t s[8];
                            tmem_ld<8>(tS + c8, s);
#pragma unroll
                            for (int c = c8; c < c8 + 8; c += 4) {
                                const float4 nr = lds4f(nr_at + 4 * c);
                                const float4 cm = lds4f(cols_at + 4 * (kCmul + c));
                                // (the score first, rounded as the references' are, then less
                                // its reference: the largest weight is 1 however large scores are)
                                const uint64_t nr2[2] = {f2(nr.x, nr.y), f2(nr.z, nr.w)};
                                [[maybe_unused]] uint64_t y[2], mq2[2];
                                if constexpr (!kOwn) {
                                    const float4 mq = lds4f(mq_at + 4 * c);
                                    mq2[0] = f2(mq.x, mq.y), mq2[1] = f2(mq.z, mq.w);
                                    const float4 sq = lds4f(sq_at + 4 * c);
                                    y[0] = mul2(ko2, f2(sq.x, sq.y));
                                    y[1] = mul2(ko2, f2(sq.z, sq.w));
                                }
                                const uint64_t cm2[2] = {f2(cm.x, cm.y), f2(cm.z, cm.w)};
                                uint64_t rd2[2];
                                if constexpr (kAgain) {
                                    const float4 rd = lds4f(cols_at + 4 * (kRedo + c));
                                    rd2[0] = f2(rd.x, rd.y), rd2[1] = f2(rd.z, rd.w);
                                }
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const int i = c / 2 + e;
                                    float y0, y1, z0, z1;
                                    const uint64_t s2 = f2(__uint_as_float(s[2 * i - c8]),
                                                           __uint_as_float(s[2 * i + 1 - c8]));
                                    if constexpr (kOwn) {  // (packed, the two would be fused)
                                        un2(s2, y0, y1);
                                        un2(nr2[e], z0, z1);
                                        y0 = __fadd_rn(__fmul_rn(y0, ks), z0);
                                        y1 = __fadd_rn(__fmul_rn(y1, ks), z1);
                                    } else {
                                        un2(fma2(fma2(s2, ks2, y[e]), mq2[e], nr2[e]), y0, y1);
                                    }
                                    if constexpr (kOwn) {
                                        y0 = seen_by(2 * i) ? y0 : neg_inf_f();
                                        y1 = seen_by(2 * i + 1) ? y1 : neg_inf_f();
                                    }
                                    y0 = ex2_mufu(y0);
                                    y1 = ex2_mufu(y1);
                                    const uint64_t p = f2(y0, y1);
                                    if constexpr (kAgain) {
                                        const uint64_t pr = mul2(p, rd2[e]);
                                        l2[i] = add2(l2[i], pr);
                                        if constexpr (!kOwn)
                                            pm2[i] = fma2(pr, vo2, pm2[i]);
                                    } else {
                                        l2[i] = add2(l2[i], p);
                                        if constexpr (!kOwn)
                                            pm2[i] = fma2(p, vo2, pm2[i]);
                                    }
                                    const uint64_t z = mul2(p, kOwn ? cm2[e] : mul2(vw2, cm2[e]));
                                    un2(z, z0, z1);
                                    top = max3(top, y0, y1);
                                    top = max3(top, z0, z1);
                                    ph[i] = pack2<W>(z0, z1);
                                    unpack2<W>(ph[i], z0, z1);
                                    un2(fma2(f2(z0, z1), f2(-kRest, -kRest),
                                             mul2(z, f2(kRest, kRest))),
                                        z0, z1);
                                    pl[i] = pack2<W>(z0, z1);
                                }
                            }
                        }
                        return top;
                    };
                    const bool busy = 32 * quarter < keys;  // some key of this warp exists
                    bool over = false;
                    if (busy) {
                        over = weights(std::false_type{}) > kTopWeight;
                    } else {
#pragma unroll
                        for (int i = 0; i < kCols / 2; ++i)
                            ph[i] = pl[i] = 0;
                    }
                    // the sums of the tile before must have read its weights
                    if (seen > summed) {
                        wait(kODone + (summed & 1), (summed >> 1) & 1);
                        ++summed;
                        tc::fence_after_sync();
                    }
                    if (kOwn && t == from && from > begin)
                        for (int at : {S::tO, S::tL})
                            scale_sums<kCols>(lanes + at + col0, nullptr, kSumUnit);
                    if (__builtin_expect(named_sync_or(kBarW + wg, 128, over), 0)) {
                        // ---- the references move: per row, the running maxima of the scores
                        // and, over the new one, of the scores with the values' scale
                        const float lv = vs > 0.0f ? log2f(vs) : neg_inf_f();
                        auto of_warps = [&](int z, int c) {  // the four warps' largest
                            const int w4 = wg * 4;
                            return fmaxf(fmaxf(wred[sb][w4][z][c], wred[sb][w4 + 1][z][c]),
                                         fmaxf(wred[sb][w4 + 2][z][c], wred[sb][w4 + 3][z][c]));
                        };
#pragma unroll 1
                        for (int i = 0; i < kCols / 4; ++i) {  // eight columns a turn, z = 0, then 1
                            const int z = i >= kCols / 8, c8 = (i - z * (kCols / 8)) * 8;
                            if (i == kCols / 8)
                                sync();
                            float to = 0.0f, m[8];
                            if (z)
                                to = fmaxf(-nref[col0 + c8 + (lane & 7)], of_warps(0, c8 + (lane & 7)));
                            uint32_t s[8];
                            tmem_ld<8>(tS + c8, s);
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                float x = score(s[c], c8 + c);
                                if (z)
                                    x = (x - __shfl_sync(0xFFFFFFFFu, to, c)) + lv;
                                m[c] = seen_by(c8 + c) ? x : neg_inf_f();
                            }
                            warp_columns<8>(m, [](float x, float y) { return fmaxf(x, y); });
                            if (lane < 8)
                                wred[sb][ww][z][c8 + lane] = m[0];
                        }
                        sync();
                        if (key < kCols) {
                            const int n = col0 + key;
                            const float ref = -nref[n];
                            const float to_ref = fmaxf(ref, of_warps(0, key));
                            // where no value has a scale yet, the second reference follows at a
                            // distance
                            const float z_old = refd[n] + (ref - to_ref);
                            const float to_z = fmaxf(fmaxf(z_old, of_warps(1, key)), -kMaxShift);
                            // a row whose weights may have overflowed starts anew with this
                            // tile: what it held weighs less than 2^-60 of what it gets
                            const bool anew = to_ref - ref > kTopShift;
                            redo[n] = anew ? 1.0f : 0.0f;
                            fl[n] = anew ? 0.0f : exp2f(ref - to_ref);
                            fo[n] = exp2f(z_old - to_z);
                            nref[n] = -to_ref;
                            refd[n] = to_z;
                            cmul[n] = exp2f(-to_z);
                        }
                        sync();
                        if (t > begin)  // the sums of the tiles before (waited for above)
                            for (int at : {S::tO, S::tL})
                                scale_sums<kCols>(lanes + at + col0, fo + col0, 1.0f);
#pragma unroll
                        for (int c = 0; c < kCols / 2; ++c) {
                            float x0, x1, m0, m1;
                            un2(l2[c], x0, x1);
                            un2(pm2[c], m0, m1);
                            const float f0 = fl[col0 + 2 * c], f1 = fl[col0 + 2 * c + 1];
                            // (a sum that is NaN stays)
                            x0 = f0 == 0.0f && x0 == x0 ? 0.0f : x0 * f0;
                            x1 = f1 == 0.0f && x1 == x1 ? 0.0f : x1 * f1;
                            m0 = f0 == 0.0f ? 0.0f : m0 * f0;
                            m1 = f1 == 0.0f ? 0.0f : m1 * f1;
                            l2[c] = f2(x0, x1);
                            pm2[c] = f2(m0, m1);
                        }
                        if (busy)
                            weights(std::true_type{});
                    }
                    // ---- the weights (own tiles: the rows of absent stages are not read)
                    if (!kOwn || busy) {
#pragma unroll
                        for (int q = 0; q < kCols / 8; ++q) {
                            sts4(p_at + 128 * q, ph[4 * q], ph[4 * q + 1], ph[4 * q + 2],
                                 ph[4 * q + 3]);
                            sts4(p_at + N * 16 + 128 * q, pl[4 * q], pl[4 * q + 1], pl[4 * q + 2],
                                 pl[4 * q + 3]);
                        }
                    }
                    fence_async_smem();
                    tc::fence_before_sync();
                    __syncwarp();
                    mbar_arrive_if(bar(kPReady), lane == 0);
                    if (!kOwn)
                        mbar_arrive_if(bar(kEmpty + st), lane == 0);
                    ++seen;
                    ring += kOwn ? (keys + 31) / 32 : 1;
                }
            };
            tiles(std::false_type{}, min(begin, g.ct), min(g.last, g.ct));
            tiles(std::true_type{}, max(begin, g.ct), max(g.last, g.ct));

            // ---- the end of the segment: sums over the keys, then the channels' results
#pragma unroll 1
            for (int z = 0; z < 2; ++z) {
                float x[kCols];
#pragma unroll
                for (int c = 0; c < kCols / 2; ++c)
                    un2(z ? pm2[c] : l2[c], x[2 * c], x[2 * c + 1]);
                warp_columns<kCols>(x, [](float u, float v) { return u + v; });
                if (lane < kCols)
                    wred[sb][ww][z][lane] = x[0];
            }
            sync();
            const bool whole = g.starts && g.ends;
            const bool poison = g.wrong || bad_page[sb];
            const int n = col0 + key;  // a row of the first lanes
            if (key < kCols && n < g.rows) {
                const int w4 = wg * 4, c = key;
                float sum = 0.0f, off = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sum += wred[sb][w4 + i][0][c];
                    off += wred[sb][w4 + i][1][c];
                }
                if (poison)
                    sum = nan_f();
                const bool none = !some || sum == 0.0f;
                const float ref = none ? kFar : -nref[n];
                const float f =
                    none ? 0.0f : exp2f(refd[n]) * (g.last > g.ct ? 1.0f : kSumUnit);
                if (whole) {
                    const float inv = none ? 0.0f : 1.0f / sum;
                    fin[sb][n] = make_float2(f * inv, poison ? nan_f() : off * inv);
                    if (a.lse)
                        a.lse[row_at[sb][n]] = none ? (poison ? nan_f() : neg_inf_f())
                                          : (ref + log2f(sum)) * 0.6931471805599453f;
                } else {
                    const int64_t at = row_at[sb][n];
                    fin[sb][n] = make_float2(f, off);
                    a.part_refs[2 * at] = ref;
                    a.part_refs[2 * at + 1] = sum;
                }
            }
            if (wt == 0 && !whole) {
                if (g.starts) {
                    meta[kOpen] = 1;
                    meta[kOpenB] = g.b;
                    meta[kOpenUnit] = g.unit;
                } else {
                    meta[kCont] = 1;
                    meta[kContEnds] = g.ends;
                }
            }
            if (seen > summed) {
                wait(kODone + (summed & 1), (summed >> 1) & 1);
                ++summed;
            }
            tc::fence_after_sync();
            sync();
            const int d = key;
            const int bad = some && any_bad[sb] ? first_bad[sb][min(d, D - 1)] : kNever;
            const int rows = g.rows;
#pragma unroll 1
            for (int c8 = 0; c8 < kCols; c8 += 8) {
                uint32_t o[8] = {0, 0, 0, 0, 0, 0, 0, 0}, rest[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (some) {
                    tmem_ld<8>(lanes + S::tO + col0 + c8, o);
                    tmem_ld<8>(lanes + S::tL + col0 + c8, rest);
                }
                if (D == 64 && quarter >= 2)
                    continue;
                if (D == 128 || d < D)
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const int n = col0 + c8 + c;
                        if (n < rows) {
                            const float2 f = fin[sb][n];
                            float x = fmaf(fmaf(__uint_as_float(rest[c]), 1.0f / kRest,
                                                __uint_as_float(o[c])),
                                           f.x, f.y);
                            if constexpr (kMasked) {
                                if (bad != kNever && meets_bad<T>(a, g, (g.r0 + n) / a.group, d, kOwnKeys))
                                    x = nan_f();
                            } else if (bad != kNever && (!a.causal || bad <= (g.r0 + n) / a.group)) {
                                x = nan_f();
                            }
                            const int64_t at = row_at[sb][n] * D + d;
                            if (whole)
                                static_cast<T *>(a.out)[at] = from_float<T>(x);
                            else
                                a.parts[at] = x;
                        }
                    }
            }
            // (what the next segment overwrites is by parity, or read no more)
            tc::fence_before_sync();
            __syncwarp();
            if (lane == 0)
                mbar_arrive(&bars[kSegEmpty + (sb)]);
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

// Joins the partials of the unit that CTA blockIdx.x of the attention began and did not finish:
// its slot 1, then slot 0 of the CTAs after it up to the one where the unit ends.  A warp takes a
// row, a lane D / 32 channels; the parts' factors are computed a lane each.
constexpr int kJoinWarps = 8;

template <typename T, int D>
__global__ void __launch_bounds__(32 * kJoinWarps)
    combine_kernel(const __grid_constant__ AttnArgs a, int N, int grid)
{
    constexpr int kV = D / 32;
    using V = std::conditional_t<kV == 4, float4, float2>;
    pdl_wait();
    const int first = blockIdx.x, lane = threadIdx.x & 31;
    const int32_t *meta = a.meta + (int64_t)first * kMeta;
    const int open = meta[kOpen], b = meta[kOpenB], unit = meta[kOpenUnit];
    if (!open)
        return;
    const int h = unit / a.row_tiles, r0 = (unit - h * a.row_tiles) * N;
    const int n = blockIdx.y * kJoinWarps + (threadIdx.x >> 5);
    if (n >= N || r0 + n >= a.rows)
        return;
    float top = kFar, sum = 0.0f, x[kV] = {};
    // 32 CTAs a turn, lane i looking at the i-th: the parts up to the one where the unit ends.
    bool more = true;
    for (int i0 = first; more && i0 < grid; i0 += 32) {
        const int i = i0 + lane;
        const int32_t *m = a.meta + (int64_t)min(i, grid - 1) * kMeta;
        const bool cont = i < grid && i > first && m[kCont];
        const uint32_t ends = __ballot_sync(0xFFFFFFFFu, cont && m[kContEnds]);
        const uint32_t upto = ends ? (2u << (__ffs(ends) - 1)) - 1u : 0xFFFFFFFFu;
        uint32_t parts = __ballot_sync(0xFFFFFFFFu, cont || i == first) & upto;
        more = ends == 0;
        const int64_t at = ((int64_t)i * 2 + (i == first)) * N + n;
        const bool mine = (parts >> lane) & 1u;
        const float ref = mine ? a.part_refs[2 * at] : kFar;
        const float part = mine ? a.part_refs[2 * at + 1] : 0.0f;
        float t = fmaxf(top, ref);
#pragma unroll
        for (int s = 16; s > 0; s >>= 1)
            t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, s));
        const float old = exp2f(top - t), f = exp2f(ref - t);
        top = t;
        sum *= old;
#pragma unroll
        for (int c = 0; c < kV; ++c)
            x[c] *= old;
        while (parts) {  // four parts' channels in flight
            V v[4];
            float pf[4], ps[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int s = parts ? __ffs(parts) - 1 : -1;
                parts &= parts - 1;
                pf[e] = __shfl_sync(0xFFFFFFFFu, f, s & 31);
                ps[e] = __shfl_sync(0xFFFFFFFFu, part, s & 31);
                const int j = i0 + s;
                v[e] = V{};
                if (s >= 0)
                    v[e] = *reinterpret_cast<const V *>(
                        a.parts + (((int64_t)j * 2 + (j == first)) * N + n) * D + kV * lane);
                else
                    pf[e] = ps[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum = fmaf(ps[e], pf[e], sum);
                const float *ve = reinterpret_cast<const float *>(&v[e]);
#pragma unroll
                for (int c = 0; c < kV; ++c)
                    x[c] = fmaf(ve[c], pf[e], x[c]);
            }
        }
    }
    const int qi = (r0 + n) / a.group, g = (r0 + n) - qi * a.group;
    const int64_t row = ((int64_t)b * a.Lq + qi) * a.Hq + h * a.group + g;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint32_t y[kV / 2];
#pragma unroll
    for (int c = 0; c < kV / 2; ++c)
        y[c] = pack2<T>(x[2 * c] * inv, x[2 * c + 1] * inv);
    uint32_t *o = reinterpret_cast<uint32_t *>(static_cast<T *>(a.out) + row * D) + kV / 2 * lane;
#pragma unroll
    for (int c = 0; c < kV / 2; ++c)
        o[c] = y[c];
    if (lane == 0 && a.lse)
        a.lse[row] = sum == 0.0f ? neg_inf_f() : (top + log2f(sum)) * 0.6931471805599453f;
}

// Rows of a row tile: the smallest width that holds a head's rows, 64 beyond that.  (64 sequences
// of 32 heads, 512 cached keys: 16 rows a head 99 us, in a tile of 32 139, of 64 175; 32 rows 139,
// in a tile of 64 184.)
int tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }

struct Workspace {
    size_t meta, refs, parts, total;
};

Workspace workspace_of(int grid, int N, int D)
{
    Workspace w;
    w.meta = 0;
    w.refs = ((size_t)grid * kMeta * 4 + 255) / 256 * 256;
    w.parts = (w.refs + (size_t)grid * 2 * N * 8 + 255) / 256 * 256;
    w.total = (w.parts + (size_t)grid * 2 * N * D * 4 + 255) / 256 * 256;
    return w;
}

int full_grid(int N) { return sm_count() * (N >= 64 ? 1 : 2); }

template <typename S, typename T, bool kMasked>
cudaError_t run(const AttnArgs &a, int grid, const CUtensorMap (&maps)[4], cudaStream_t s)
{
    static PerDevice ready;
    cudaError_t e = ready.once([] {
        // the roles' shares of registers must not add up to more than the launch gives
        cudaFuncAttributes f;
        const cudaError_t got = cudaFuncGetAttributes(&f, attention_kernel<S, T, kMasked>);
        if (got != cudaSuccess || f.numRegs < S::regs)
            return got != cudaSuccess ? got : cudaErrorInvalidKernelImage;
        return cudaFuncSetAttribute(attention_kernel<S, T, kMasked>,
                                    cudaFuncAttributeMaxDynamicSharedMemorySize, S::smem);
    });
    if (e != cudaSuccess)
        return e;
    e = launch(attention_kernel<S, T, kMasked>, dim3(grid), dim3(S::threads), S::smem, s, true,
                           a, maps[0], maps[1], maps[2], maps[3]);
    if (e != cudaSuccess)
        return e;
    return launch(combine_kernel<T, S::D>, dim3(grid, (S::N + kJoinWarps - 1) / kJoinWarps),
                  dim3(32 * kJoinWarps), 0, s, true, a, S::N, grid);
}

template <int D, typename T, bool kMasked>
cudaError_t run_rows(const AttnArgs &a, int N, int grid, const CUtensorMap (&maps)[4],
                     cudaStream_t s)
{
    return N == 16   ? run<Shape<D, 16>, T, kMasked>(a, grid, maps, s)
           : N == 32 ? run<Shape<D, 32>, T, kMasked>(a, grid, maps, s)
                     : run<Shape<D, 64>, T, kMasked>(a, grid, maps, s);
}

// The checks and the launches of both entry points.
template <bool kMasked>
fdllm_status attend(const void *q, const int64_t *q_strides, int dtype, int B, int Lq, int Hq,
                    const fdllm_cache *cache, const int32_t *block_table, int max_pages,
                    const int32_t *cache_lens, const void *k_new, const int64_t *k_strides,
                    const void *v_new, const int64_t *v_strides, int Ln, const int32_t *new_lens,
                    int causal, const uint32_t *sees, double scale, void *out, float *out_lse,
                    void *workspace, size_t workspace_bytes, void *stream)
{
    AttnArgs a = {};
    const fdllm_status st = check_cache(cache, a.c);
    if (st != FDLLM_OK)
        return st;
    if (!check_table(block_table, B, max_pages, a.c.page_shift, a.c.heads) || !cache_lens ||
        !check_queries(q, q_strides, dtype, B, Lq, Hq, a.c.heads) || Ln < 0 ||
        Ln >= (1 << 30) || (Ln > 0 && (!k_new || !v_new || !k_strides || !v_strides)) ||
        (causal != 0 && causal != 1) || (kMasked && Ln > 0 && !sees) || !std::isfinite(scale) || !out)
        return FDLLM_ERR_ARG;
    const int64_t none[1] = {0};
    if (!aligned16(q, q_strides, 3, 2) || !aligned16(out, none, 0, 2) ||
        (Ln > 0 && (!aligned16(k_new, k_strides, 3, 2) || !aligned16(v_new, v_strides, 3, 2))))
        return FDLLM_ERR_ALIGN;
    const int64_t rows = (int64_t)Lq * (Hq / a.c.heads);
    const int N = tile_rows(rows), D = a.c.D;
    const int most = full_grid(N);
    const Workspace ws = workspace_of(most, N, D);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
        workspace_bytes < ws.total)
        return FDLLM_ERR_WORKSPACE;
    a.table = block_table;
    a.max_pages = max_pages;
    a.lens = cache_lens;
    a.q = q;
    a.qs = strides3(q_strides);
    a.B = B;
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
    a.sees = sees;
    a.sees_words = (int)(((int64_t)Ln + 31) / 32);
    a.scale = (float)(scale * 1.4426950408889634);
    a.out = out;
    a.lse = out_lse;
    a.rows = (int)rows;
    a.row_tiles = (int)((rows + N - 1) / N);
    if ((int64_t)a.c.heads * a.row_tiles >= ((int64_t)1 << 31))
        return FDLLM_ERR_ARG;
    uint8_t *w = static_cast<uint8_t *>(workspace);
    a.meta = reinterpret_cast<int32_t *>(w + ws.meta);
    a.part_refs = reinterpret_cast<float *>(w + ws.refs);
    a.parts = reinterpret_cast<float *>(w + ws.parts);
    // No more CTAs than the call can have tiles.
    const int64_t slots = (int64_t)max_pages << a.c.page_shift;
    const int64_t tiles = (slots + kKeys - 1) / kKeys + ((int64_t)Ln + kKeys - 1) / kKeys;
    int64_t bound = most;
    if ((int64_t)a.c.heads * a.row_tiles < most && (int64_t)a.c.heads * a.row_tiles * B < most)
        bound = (int64_t)a.c.heads * a.row_tiles * B * tiles;
    const int grid = (int)(bound < most ? bound : most);
    CUtensorMap maps[4] = {};  // the cache's keys and values, the block's own
    a.status = cache_status_word();
    if (!a.status || !make_cache_maps(a.c, &maps[0], &maps[1]))
        return FDLLM_ERR_CUDA;
    a.mapped = Ln > 0 &&
               make_rows_map(&maps[2], k_new, a.ks, B, Ln, a.c.heads, D, 64, true) &&
               make_rows_map(&maps[3], v_new, a.vs, B, Ln, a.c.heads, D, D, false);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf = dtype == FDLLM_BF16;
    const cudaError_t e =
        D == 128 ? (bf ? run_rows<128, __nv_bfloat16, kMasked>(a, N, grid, maps, s)
                       : run_rows<128, __half, kMasked>(a, N, grid, maps, s))
                 : (bf ? run_rows<64, __nv_bfloat16, kMasked>(a, N, grid, maps, s)
                       : run_rows<64, __half, kMasked>(a, N, grid, maps, s));
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

}  // namespace
}  // namespace fdllm
