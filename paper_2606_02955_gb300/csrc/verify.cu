// verify.cu -- fdllm_verify_draft: drafted tokens taken or rejected by the target's probabilities and
// given random numbers, and the token that follows the taken ones.
//
// Mathematics.  p_j = softmax(target row j / T) after node j, q_j the draft's likewise.
//   a chain drawn from q: node j + 1 with token d is taken iff u q_j(d) < p_j(d); where the first is
//   not, after node c, the next token is drawn from max(p_c - q_c, 0), else from the last p_c.
//   tokens that were not drawn (a tree's, or a chain's without the draft's logits): the children of c
//   in turn, child k taken iff u (1 - sum of the p_c of those before it) < p_c(d_k); where none
//   is, the next token is drawn from p_c without the children's tokens.
// A token is drawn from weights r(v) as argmax r(v) / E(v), E given (exponential variables): r needs
// no norm, and no sum over the vocabulary has to be exact to the last token's share.
//
// Two kernels.  The first takes every row's maximum and sum (or its largest value) in one pass, in
// parts that no CTA waits for; the second joins the parts, walks the nodes and draws the next token,
// reading again only the one or two rows it is drawn from.  A kernel that walked as sums came and left out
// the rows behind a rejection took 72 us and more where these take 57 (64 chains of nine): decisions
// come 10 us and more behind the copies, and copies under way are not taken back.  Trees are another
// matter where few of their many rows are on the path: there the second kernel comes alone, and its
// clusters sum the rows as their walk comes to them.
//
// Bound by HBM where rows are many and long: 64 chains of up to nine rows of 126464 bf16 values and the
// draft's rows, 57 us: 45 of the first kernel (243 MB, 5.4 TB/s, half of the issue slots taken), the
// rest of the draw (63 MB), which the first does not hide.  A walk by latencies, about 3 us a turn (8
// trees of 48 nodes of 126464 values 14.6 us in all).  By two launches and the draw's chain (parts,
// decisions, weights, the cluster's best) where they are few: a chain of five rows of 32000 values 9 us.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "vocab_rows.cuh"

namespace fdllm {
namespace {

namespace cg = cooperative_groups;

constexpr int kMaxNodes = FDLLM_MAX_L;
constexpr int kMathWarps = 16;
constexpr int kMath = 32 * kMathWarps;
constexpr int kChunk = 65536;  // bytes of a stage (six stages of half as many: 61 us for 59)
constexpr int kStages = 3;
constexpr int kChunkVecs = kChunk / 16;
// Rows up to this many bytes: a few warps each, without the ring, whose beginning and end cost more than
// their copies hide (14 trees of 53 rows of 23 KB, the whole call: 14.8 us, with the ring 24.8).
constexpr int kSmallRow = 32768;
// Vectors of a lane in such a row, about (33 chains of 51 rows of 2088 values 11.5 us, with four vectors
// 13.5, with sixteen 10.8; 8 of nine of 8000 9.1, 9.2 and 9.9; 14 trees of 53 of 11500 16.7, 16.6 and 13.4).
constexpr int kSmallVecs = 8;
constexpr int kDraw = 512;       // threads of a CTA of the walk and the draw (256: 69 us for 58)
constexpr int kMaxRanks = 8;     // CTAs of a cluster of them

struct VerifyArgs {
    const void *target;       // [B, M, V]
    const void *draft;        // [B, M - 1, V] or null
    int64_t t_batch, t_row, d_batch, d_row;  // strides, in values
    int B, M, V;
    const int32_t *tokens;    // [B, M]
    const int32_t *parents;   // [B, M] or null: a chain
    const int32_t *lens;      // [B] or null: M
    int greedy;
    float ct, cd;             // log2(e) / temperature, of the target's rows and of the draft's
    const float *uniform;     // [B, M]
    const float *noise;       // [B, V]
    int32_t *out_tokens;      // [B, M]
    int32_t *out_nodes;       // [B, M]
    int32_t *out_n;           // [B]
    UnitPartial *parts;       // [B, M] of the target's rows, [B, M - 1] of the draft's; each `per` long
    int per;                  // parts of a row
    int pieces, piece_vecs;   // pieces of a row, vectors of one
    int turn, turn_most;      // rows of a turn of the walk at first, and at most
    uint32_t *status;         // sticky: a bounded wait gave up, in whatever call
    uint32_t *gave_up;        // [streams] one did in that CTA of the first kernel
    int streams;
};

__device__ __forceinline__ int nodes_of(const VerifyArgs &a, int b)
{
    return a.lens ? min(max(__ldg(a.lens + b), 1), a.M) : a.M;
}

// Where row j of sequence b is: of the target, or of the draft.
struct RowAt {
    int64_t part;  // its parts
    const uint8_t *p;
};

template <typename T>
__device__ __forceinline__ RowAt row_at(const VerifyArgs &a, int b, int j, bool of_draft)
{
    RowAt r;
    r.part = (of_draft ? (int64_t)a.B * a.M + (int64_t)b * (a.M - 1) + j : (int64_t)b * a.M + j) * a.per;
    const int64_t at = of_draft ? b * a.d_batch + j * a.d_row : b * a.t_batch + j * a.t_row;
    r.p = static_cast<const uint8_t *>(of_draft ? a.draft : a.target) + at * (int64_t)sizeof(T);
    return r;
}

// A thread's largest value and its first index; `nan` where a value is one.
struct Largest {
    float m = -INFINITY;
    uint32_t first = kNoIdx;
    float nan = -INFINITY;

    template <typename T, int N>
    __device__ __forceinline__ void add(const uint4 (&x)[N], const int (&i)[N])
    {
        constexpr int E = 16 / sizeof(T);
        float top = -INFINITY;
        uint4 r = x[0];
        int at = i[0];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float y = vector_most<T>(x[n]);
            nan = fmax_nan(nan, y);
            if (y > top) {
                top = y;
                r = x[n];
                at = i[n];
            }
        }
        if (top > m) {
            float y[E];
            widen<T>(r, y);
#pragma unroll
            for (int e = E - 1; e >= 0; --e)
                if (y[e] == top)
                    first = at + e;
            m = top;
        }
    }
    __device__ __forceinline__ void add(float x, int i)
    {
        nan = fmax_nan(nan, x);
        if (x > m || (x == m && (uint32_t)i < first)) {
            m = x;
            first = i;
        }
    }
};

// What a warp makes of its share of a row: its part of the sum, or its largest value (S then 1, or
// NaN, and 0 where there is no finite value).
template <typename T, bool kGreedy>
struct Share {
    Summed s;
    Largest l;
    template <int N>
    __device__ __forceinline__ void add(const uint4 (&x)[N], const int (&i)[N], float c)
    {
        if constexpr (kGreedy)
            l.template add<T, N>(x, i);
        else
            s.template add<T, N>(x, c);
    }
    // The values before the row's first whole vector and behind its last.
    __device__ __forceinline__ void add_ends(const RowSpan<T> &r, float c)
    {
        const int lane = threadIdx.x & 31;
        const int i = lane < 8 ? lane : r.tail() + lane - 8;
        if (!(lane < 8 ? i < r.head : i < r.V && lane < 16))
            return;
        const float x = to_float(r.row[i]);
        if constexpr (kGreedy) {
            l.add(x, i);
        } else {
            s.settle(c);
            s.z.add(x, c);
        }
    }
    __device__ __forceinline__ UnitPartial join(float c)
    {
        UnitPartial p;
        p.pad = 0;
        if constexpr (kGreedy) {
            p.M = warp_most(l.m);
            p.idx = __reduce_min_sync(0xFFFFFFFFu, l.m == p.M ? l.first : kNoIdx);
            const bool bad = __any_sync(0xFFFFFFFFu, l.nan != l.nan);
            p.S = bad ? nan_f() : p.M == -INFINITY ? 0.0f : 1.0f;
        } else {
            s.settle(c);
            const ExpSum z = warp_sum(s.z, c);
            p.M = z.m;
            p.S = z.z;
            p.idx = kNoIdx;
        }
        return p;
    }
};

// ---- Rows of up to kSmallRow bytes: a.per warps each, every one with a part of its own.
template <typename T, bool kGreedy>
__global__ void __launch_bounds__(256) verify_small_kernel(const __grid_constant__ VerifyArgs a)
{
    constexpr int E = 16 / sizeof(T);
    pdl_wait();
    if (threadIdx.x == 0)
        pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int64_t targets = (int64_t)a.B * a.M, rows = targets + (a.draft ? (int64_t)a.B * (a.M - 1) : 0);
    const int64_t step = (int64_t)gridDim.x * 8;
    for (int64_t w = blockIdx.x * 8ll + (threadIdx.x >> 5); w < rows * a.per; w += step) {
        const int64_t row = w / a.per;
        const int share = (int)(w - row * a.per);
        const bool of_draft = row >= targets;
        const int64_t at = of_draft ? row - targets : row;
        const int per = of_draft ? a.M - 1 : a.M;
        const int b = (int)(at / per), j = (int)(at - (int64_t)b * per);
        if (j >= nodes_of(a, b) - (of_draft ? 1 : 0))
            continue;
        const float c = of_draft ? a.cd : a.ct;
        const RowAt where = row_at<T>(a, b, j, of_draft);
        const RowSpan<T> r(reinterpret_cast<const T *>(where.p), a.V);
        Share<T, kGreedy> s;
        constexpr uint32_t kPad = no_values<T>();
        for (int v = 32 * share + lane; v < r.vecs; v += 128 * a.per) {
            uint4 x[4];
            int i[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int at = v + 32 * a.per * n;
                x[n] = at < r.vecs ? r.vectors()[at] : make_uint4(kPad, kPad, kPad, kPad);
                i[n] = r.head + at * E;
            }
            s.template add<4>(x, i, c);
        }
        if (share == 0)
            s.add_ends(r, c);
        const UnitPartial p = s.join(c);
        if (lane == 0)
            a.parts[where.part + share] = p;
    }
}

// ---- Longer rows: pieces of them stream through a ring of shared memory, filled by bulk copies.
// Every warp leaves its own part of a piece: no warp waits for another but through the ring.  Pieces go
// to CTAs in turn; ranges of equal bytes, one to a CTA, end together, and took 64 us for 57: the
// CTAs that end early leave their SMs to the draw's, which bring the noise in meanwhile.
struct Stage {
    uint32_t n;     // vectors, 0: no more
    int32_t at;     // index in the row of their first value
    uint32_t last;  // 1: the piece ends here, 2: and the row
    float c;
    int64_t part;   // the piece's parts
    const void *row;
};

struct StreamShared {
    uint64_t full[kStages], empty[kStages];
    Stage stage[kStages];
};
constexpr int kMostStreams = 512;  // CTAs of it (the workspace's size does not ask for the GPU's)
constexpr int kStreamSmem = kStages * kChunk + (int)sizeof(StreamShared);

template <typename T, bool kGreedy>
__global__ void __launch_bounds__(kMath + 32, 1)
    verify_stream_kernel(const __grid_constant__ VerifyArgs a)
{
    constexpr int E = 16 / sizeof(T);
    constexpr int kPer = kChunkVecs / kMath;
    extern __shared__ __align__(128) uint8_t ring[];
    StreamShared &sm = *reinterpret_cast<StreamShared *>(ring + kStages * kChunk);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], kMathWarps);
        }
        fence_mbar_init();
    }
    pdl_wait();
    if (threadIdx.x == 0) {
        a.gave_up[blockIdx.x] = 0;
        pdl_launch_dependents();
    }
    __syncthreads();
    // What a wait that gave up leaves undone, the second kernel learns from the call's own word: the
    // sticky one may have been asked for, and cleared, in between.
    auto wait = [&](uint64_t *bar, uint32_t parity, uint64_t limit_ns) {
        const bool done = mbar_wait(bar, parity, a.status, limit_ns);
        if (!done)
            a.gave_up[blockIdx.x] = 1;
        return done;
    };
    if (warp == kMathWarps) {
        // ------------------------------------------------------------ the copying lane
        if (lane != 0)
            return;
        const uint64_t policy = make_evict_first_policy();
        const uint32_t kinds = a.draft ? 2 : 1;
        const uint32_t units = (uint32_t)a.B * a.M * kinds * a.pieces;
        uint32_t k = 0;
        bool alive = true;
        for (uint32_t u = blockIdx.x; u < units && alive; u += gridDim.x) {
            // nodes first, so that all sequences' early rows come first
            const uint32_t row = u / a.pieces, piece = u - row * a.pieces;
            const uint32_t bj = row / kinds, of_draft = row - bj * kinds;
            const int j = (int)(bj / a.B), b = (int)(bj - (uint32_t)j * a.B);
            if (j >= nodes_of(a, b) - (int)of_draft)
                continue;
            const RowAt where = row_at<T>(a, b, j, of_draft);
            const RowSpan<T> r(reinterpret_cast<const T *>(where.p), a.V);
            const int end = (int)piece + 1 < a.pieces ? (int)(piece + 1) * a.piece_vecs : r.vecs;
            for (int v = piece * a.piece_vecs; v < end; v += kChunkVecs, ++k) {
                const uint32_t s = k % kStages;
                if (k >= kStages && !wait(&sm.empty[s], (k / kStages - 1) & 1, kWaitLimitNs)) {
                    alive = false;
                    break;
                }
                const uint32_t n = min(kChunkVecs, end - v);
                Stage st;
                st.n = n;
                st.at = r.head + v * E;
                st.last = v + (int)n < end ? 0 : (int)piece + 1 < a.pieces ? 1 : 2;
                st.c = of_draft ? a.cd : a.ct;
                st.part = where.part + piece * kMathWarps;
                st.row = r.row;
                sm.stage[s] = st;
                mbar_arrive_expect_tx(&sm.full[s], n * 16);
                bulk_copy_g2s_hint(ring + s * kChunk, r.vectors() + v, n * 16, &sm.full[s], policy);
            }
        }
        if (alive) {
            const uint32_t s = k % kStages;
            if (k < kStages || wait(&sm.empty[s], (k / kStages - 1) & 1, kWaitLimitNs)) {
                sm.stage[s].n = 0;
                mbar_arrive(&sm.full[s]);
            } else {
                alive = false;
            }
        }
        // nothing may land in this CTA's memory after it has gone
        // (the stage that holds the end had its last copy taken)
        const uint32_t most = alive ? kStages - 1 : kStages;
        for (uint32_t i = k > most ? k - most : 0; i < k; ++i)
            wait(&sm.full[i % kStages], (i / kStages) & 1, kDrainLimitNs);
        return;
    }
    // ---------------------------------------------------------------- the counting warps
    constexpr uint32_t kPad = no_values<T>();
    Share<T, kGreedy> sum;
    for (uint32_t k = 0;; ++k) {
        const uint32_t s = k % kStages;
        if (!wait(&sm.full[s], (k / kStages) & 1, kWaitLimitNs))
            return;
        const Stage &st = sm.stage[s];
        const uint32_t vecs = st.n, last = st.last;
        if (vecs == 0)
            return;
        const float c = st.c;
        const int64_t part = st.part;
        const T *row = static_cast<const T *>(st.row);
        const uint4 *buf = reinterpret_cast<const uint4 *>(ring + s * kChunk);
        uint4 x[kPer];
        int i[kPer];
        if (vecs == kChunkVecs) {
#pragma unroll
            for (int n = 0; n < kPer; ++n)
                x[n] = buf[threadIdx.x + n * kMath];
        } else {
#pragma unroll
            for (int n = 0; n < kPer; ++n) {
                const uint32_t v = threadIdx.x + n * kMath;
                x[n] = v < vecs ? buf[v] : make_uint4(kPad, kPad, kPad, kPad);
            }
        }
#pragma unroll
        for (int n = 0; n < kPer; ++n)
            i[n] = st.at + (threadIdx.x + n * kMath) * E;
        __syncwarp();
        if (lane == 0)
            mbar_arrive(&sm.empty[s]);
        sum.template add<kPer>(x, i, c);
        if (!last)
            continue;
        if (last == 2 && warp == 0)
            sum.add_ends(RowSpan<T>(row, a.V), c);
        const UnitPartial p = sum.join(c);
        if (lane == 0)
            a.parts[part + warp] = p;
        sum = Share<T, kGreedy>();
    }
}

// ---- The walk.
// A row's parts joined.
struct RowSum {
    ExpSum z;
    uint32_t first = kNoIdx;

    __device__ __forceinline__ void take(const int4 &r, bool greedy, float c)
    {
        ExpSum o;
        o.m = __int_as_float(r.x);
        o.z = __int_as_float(r.y);
        if (greedy) {
            if (o.m > z.m || (o.m == z.m && (uint32_t)r.z < first))
                first = (uint32_t)r.z;
            z.m = fmaxf(z.m, o.m);
            z.z += o.z;
        } else {
            z.merge(o, c);
        }
    }
    __device__ __forceinline__ void join_warp(bool greedy, float c)
    {
        if (greedy) {
            const float top = warp_most(z.m);
            first = __reduce_min_sync(0xFFFFFFFFu, z.m == top ? first : kNoIdx);
            z.m = top;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                z.z += __shfl_xor_sync(0xFFFFFFFFu, z.z, o);
        } else {
            z = warp_sum(z, c);
        }
    }
};

__device__ __forceinline__ bool usable(const ExpSum &z)
{
    return z.z > 0.0f && z.z <= FLT_MAX && finite_f(z.m);
}

constexpr int kNone = 0, kBad = -1;  // choices that are no child

// A sequence's nodes, and what the walk finds out about them: arrays of M in shared memory.
struct Nodes {
    ExpSum *of, *less;   // row sums: the target's, the draft's
    float *uniform;
    float *x, *y;        // the logits of its token after its parent: target's, draft's
    int *token;
    uint32_t *first;     // greedy: the largest logit's index
    short *parent;       // -1: none
    short *choice;
    short *path;
    uint32_t *gone;      // a bit for each token of the slice: those tried after the last node
    static constexpr int kBytes = 2 * 8 + 5 * 4 + 3 * 2;  // of a node

    __device__ __forceinline__ Nodes(uint8_t *p, int M)
    {
        M = (M + 7) / 8 * 8;
        of = reinterpret_cast<ExpSum *>(p);
        less = of + M;
        uniform = reinterpret_cast<float *>(less + M);
        x = uniform + M;
        y = x + M;
        token = reinterpret_cast<int *>(y + M);
        first = reinterpret_cast<uint32_t *>(token + M);
        parent = reinterpret_cast<short *>(first + M);
        choice = parent + M;
        path = choice + M;
        gone = reinterpret_cast<uint32_t *>(path + M);
    }
};
inline size_t draw_smem(int M, int V, int ranks, bool greedy)
{
    return (size_t)(M + 7) / 8 * 8 * Nodes::kBytes +
           (greedy ? 0 : (size_t)((V + ranks - 1) / ranks + 31) / 32 * 4);
}

// The sums of a sequence's rows, of the target's n and of the draft's n - 1: a thread a row where a row
// is a few parts, else a warp, with the first parts of kAhead rows on their way at once.
template <typename T>
__device__ __forceinline__ void sum_rows(const VerifyArgs &a, const Nodes &s, int b, int n)
{
    constexpr int kAhead = 4;
    const int rows = a.draft ? 2 * n - 1 : n;
    auto keep = [&](int r, const RowSum &x) {
        if (r < n) {
            s.of[r] = x.z;
            s.first[r] = x.first;
        } else {
            s.less[r - n] = x.z;
        }
    };
    auto parts = [&](int r) {
        return reinterpret_cast<const int4 *>(a.parts + (r < n ? row_at<T>(a, b, r, false).part
                                                               : row_at<T>(a, b, r - n, true).part));
    };
    if (a.per <= 8) {
        for (int r = threadIdx.x; r < rows; r += kDraw) {
            RowSum x;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < a.per)
                    x.take(__ldcg(parts(r) + i), a.greedy, r < n ? a.ct : a.cd);
            keep(r, x);
        }
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int r0 = warp; r0 < rows; r0 += kAhead * (kDraw / 32)) {
        int4 p[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int r = r0 + k * (kDraw / 32);
            if (r < rows && lane < a.per)
                p[k] = __ldcg(parts(r) + lane);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int r = r0 + k * (kDraw / 32);
            if (r >= rows)
                break;
            const float c = r < n ? a.ct : a.cd;
            RowSum x;
            if (lane < a.per)
                x.take(p[k], a.greedy, c);
            for (int i = lane + 32; i < a.per; i += 32)
                x.take(__ldcg(parts(r) + i), a.greedy, c);
            x.join_warp(a.greedy, c);
            if (lane == 0)
                keep(r, x);
        }
    }
}

// p of node j's token after its parent c, q of it; 0 for a token out of the vocabulary.
__device__ __forceinline__ float p_of_node(const VerifyArgs &a, const Nodes &s, int c, int j)
{
    const bool inside = s.token[j] >= 0 && s.token[j] < a.V;
    return inside ? ex2_mufu((s.x[j] - s.of[c].m) * a.ct) / s.of[c].z : 0.0f;
}
__device__ __forceinline__ float q_of_node(const VerifyArgs &a, const Nodes &s, int c, int j)
{
    const bool inside = s.token[j] >= 0 && s.token[j] < a.V;
    return inside ? ex2_mufu((s.y[j] - s.less[c].m) * a.cd) / s.less[c].z : 0.0f;
}

// Which child of node c is taken, kNone, or kBad where a row of c is unusable.  Of a chain, by a thread:
__device__ __forceinline__ int decide_chain(const VerifyArgs &a, const Nodes &s, int c, int n)
{
    const int j = c + 1;
    if (!usable(s.of[c]) || (a.draft && j < n && !usable(s.less[c])))
        return kBad;
    if (j >= n)
        return kNone;
    if (a.greedy)
        return (uint32_t)s.token[j] == s.first[c] ? j : kNone;
    const float p = p_of_node(a, s, c, j);
    const double u = s.uniform[j];
    return u * (a.draft ? (double)q_of_node(a, s, c, j) : 1.0) < (double)p ? j : kNone;
}

// Of a tree, by a warp:
__device__ __forceinline__ int decide(const VerifyArgs &a, const Nodes &s, int c, int n)
{
    const int lane = threadIdx.x & 31;
    if (!usable(s.of[c]))
        return kBad;
    double left = 1.0;
    for (int j0 = c + 1; j0 < n; j0 += 32) {
        const int j = j0 + lane;
        const bool child = j < n && s.parent[j] == c;
        uint32_t kids = __ballot_sync(0xFFFFFFFFu, child);
        if (!kids)
            continue;
        const int d = child ? s.token[j] : -1;
        if (a.greedy) {
            const uint32_t hit = __ballot_sync(0xFFFFFFFFu, child && (uint32_t)d == s.first[c]);
            if (hit)
                return j0 + __ffs(hit) - 1;
            continue;
        }
        float p = child ? p_of_node(a, s, c, j) : 0.0f;
        // a token that was tried before counts 0: among these 32, and among those before them
        if (__match_any_sync(0xFFFFFFFFu, d) & kids & ((1u << lane) - 1))
            p = 0.0f;
        for (int i0 = c + 1; i0 < j0; i0 += 32) {
            const bool kin = s.parent[i0 + lane] == c;
            const int e = s.token[i0 + lane];
            for (uint32_t bits = __ballot_sync(0xFFFFFFFFu, kin); bits; bits &= bits - 1)
                if (__shfl_sync(0xFFFFFFFFu, e, __ffs(bits) - 1) == d)
                    p = 0.0f;
        }
        const float u = child ? s.uniform[j] : 0.0f;
        for (; kids; kids &= kids - 1) {
            const int k = __ffs(kids) - 1;
            const float pk = __shfl_sync(0xFFFFFFFFu, p, k), uk = __shfl_sync(0xFFFFFFFFu, u, k);
            if ((double)uk * left < (double)pk)
                return j0 + k;
            left -= pk;
        }
    }
    return kNone;
}

// ---- Trees of many nodes: the rows on the path alone are read, each by the whole cluster.
constexpr int kTurn = 8;  // rows of a turn at most
// Rows are read along the way where all of them are this many bytes: long ones (beyond kSmallRow), short
// ones.  In bf16: 8 trees of 48 nodes of 126464 values 14.6 us (all rows first: 34.5), 16 of 60 of 32000
// 13.5 (26.4), one of 48 of 126464 (12 MB) 11.2 (18.2), 64 of 40 of 11500 20 (30); but 8 of 16 of 32000
// (8 MB) 13 (12), 14 of 53 of 11500 (17 MB) 16.8 (15.2).  Where paths are long the turns add up: 8 trees
// that are chains of 48, every node taken, are 52 us (22), with two rows a turn throughout more.
constexpr int64_t kWalkLong = 12000000, kWalkShort = 40000000;
// Bytes of a row that a CTA is worth (half and twice as many are alike; four times: 16 trees of 60 of 32000
// values 15.2 us for 13.8, 64 of 40 of 11500 19.1 for 18.1).
constexpr int kWalkShare = 8192;
// Of a CTA's share of a turn's rows, and twice that where it went well (half: one tree of 48 of 126464 20.6
// us for 15.7, 64 of 60 of 19000 23.4 for 21.2, 64 of 40 of 11500 17.4 for 18.1; twice: 8 of 48 of 126464
// 17.1 for 14.7).
constexpr int kTurnBytes = 1 << 16;

struct WalkShared {
    int4 part[kDraw / 32];                // of a warp's share of its row
    int4 slot[2][kTurn][kMaxRanks];       // of a CTA's, by the turn's parity
};

// The first child of node c, -1: none.  By a warp.
__device__ __forceinline__ int first_child(const Nodes &s, int c, int n)
{
    const int lane = threadIdx.x & 31;
    for (int j0 = c + 1; j0 < n; j0 += 32) {
        const uint32_t kids = __ballot_sync(0xFFFFFFFFu, j0 + lane < n && s.parent[j0 + lane] == c);
        if (kids)
            return j0 + __ffs(kids) - 1;
    }
    return -1;
}

// The walk by turns: the row of the node that it has come to and, on the way to a drafter's best guess,
// those of its first child, that one's first child and so on, summed at once by warps of every CTA.
// Where it went all the way down, the next turn takes twice as many.  A turn waits for its rows and for the
// other CTAs' sums of them; nothing of a row is kept, the draw finds the last one in the L2.
template <typename T, bool kGreedy>
__device__ __forceinline__ void walk(const VerifyArgs &a, const Nodes &s, WalkShared &sm, int b, int n,
                                     const cg::cluster_group &cluster, int &taken, int &failed)
{
    constexpr int E = 16 / sizeof(T), kWarps = kDraw / 32, kEight = 8;
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int at = 0, len = 0, most = a.turn;
    for (uint32_t turn = 0;; ++turn) {
        int node[kTurn], rows = 1, mine = at;
        node[0] = at;
#pragma unroll
        for (int g = 1; g < kTurn; ++g) {
            node[g] = g < most && node[g - 1] >= 0 ? first_child(s, node[g - 1], n) : -1;
            rows += node[g] >= 0;
        }
        const int g = warp % rows;
#pragma unroll
        for (int i = 1; i < kTurn; ++i)
            mine = g == i ? node[i] : mine;
        const RowSpan<T> r(reinterpret_cast<const T *>(row_at<T>(a, b, mine, false).p), a.V);
        const int per = (r.vecs + ranks - 1) / ranks;
        const int lo = min(r.vecs, rank * per), hi = min(r.vecs, lo + per);
        const int wide = 32 * ((kWarps - g + rows - 1) / rows);  // threads of the row
        Share<T, kGreedy> share;
        for (int v = lo + (warp / rows) * 32 + lane; v < hi; v += kEight * wide) {
            constexpr uint32_t kPad = no_values<T>();
            uint4 x[kEight];
            int i[kEight];
#pragma unroll
            for (int q = 0; q < kEight; ++q) {
                const int w = v + q * wide;
                x[q] = w < hi ? r.vectors()[w] : make_uint4(kPad, kPad, kPad, kPad);
                i[q] = r.head + w * E;
            }
            share.template add<kEight>(x, i, a.ct);
        }
        if (rank == 0 && warp < rows)
            share.add_ends(r, a.ct);
        const UnitPartial p = share.join(a.ct);
        if (lane == 0)
            sm.part[warp] = make_int4(__float_as_int(p.M), __float_as_int(p.S), (int)p.idx, 0);
        __syncthreads();
        if (warp < rows) {
            RowSum x;
            if (warp + lane * rows < kWarps)
                x.take(sm.part[warp + lane * rows], kGreedy, a.ct);
            x.join_warp(kGreedy, a.ct);
            if (lane < ranks)
                *cluster.map_shared_rank(&sm.slot[turn & 1][warp][rank], lane) =
                    make_int4(__float_as_int(x.z.m), __float_as_int(x.z.z), (int)x.first, 0);
        }
        cluster_arrive();
        cluster_wait();
        if (warp < rows) {
            RowSum x;
            if (lane < ranks)
                x.take(sm.slot[turn & 1][warp][lane], kGreedy, a.ct);
            x.join_warp(kGreedy, a.ct);
            if (lane == 0) {
                s.of[mine] = x.z;
                s.first[mine] = x.first;
            }
            __syncwarp();
            const int to = decide(a, s, mine, n);
            if (lane == 0)
                s.choice[mine] = (short)to;
        }
        __syncthreads();
        most = min(a.turn_most, 2 * most);
#pragma unroll
        for (int i = 0; i < kTurn; ++i) {
            if (i >= rows)
                break;
            if (node[i] != at) {
                most = a.turn;
                break;
            }
            if (threadIdx.x == 0)
                s.path[len] = (short)at;
            const int to = s.choice[at];
            if (to <= 0) {
                if (threadIdx.x == 0) {
                    taken = len;
                    failed = to == kBad;
                }
                return;
            }
            at = to;
            ++len;
        }
    }
}

// Clusters of CTAs, one to a sequence: the walk, in each CTA; then the draw, each CTA a slice of the
// vocabulary.  What the call was given is read, and the noise brought to the L2, while the rows'
// sums are still under way: it was there before their kernel began.  kWalk: no kernel came before,
// the rows are summed as the walk comes to them.
template <typename T, bool kWalk>
__global__ void __launch_bounds__(kDraw, kWalk ? 1 : 2)
    verify_draw_kernel(const __grid_constant__ VerifyArgs a)
{
    constexpr int E = 16 / sizeof(T);
    __shared__ int taken, failed, undone;
    __shared__ unsigned long long of_cta[kMaxRanks];
    __shared__ uint2 best[kDraw / 32];
    extern __shared__ __align__(16) uint8_t dynamic[];
    const Nodes s(dynamic, a.M);
    uint32_t *const gone = s.gone;
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = blockIdx.x / ranks, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int slice = ((a.V + ranks - 1) / ranks + 31) / 32 * 32;
    const int v0 = min(a.V, rank * slice), v1 = min(a.V, v0 + slice);
    const int64_t base = (int64_t)b * a.M;
    const float *noise = a.noise + (int64_t)b * a.V;
    cluster_arrive_relaxed();  // (that this CTA is there; waited for where another writes to it)
    if constexpr (kWalk) {
        pdl_wait();
        const uint8_t *root = row_at<T>(a, b, 0, false).p;
        for (int v = v0 + tid * (128 / (int)sizeof(T)); v < v1; v += kDraw * (128 / (int)sizeof(T)))
            asm volatile("prefetch.global.L2 [%0];" ::"l"(root + (int64_t)v * sizeof(T)));
    }
    if (!a.greedy) {
        for (int i = tid; i < slice / 32; i += kDraw)
            gone[i] = 0;
        for (int v = v0 + tid * 32; v < v1; v += kDraw * 32)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(noise + v));
    }
    const int n = nodes_of(a, b);
    for (int j = tid; j < n; j += kDraw) {
        const int p = j == 0 ? -1 : a.parents ? a.parents[base + j] : j - 1;
        const int d = a.tokens[base + j];
        s.parent[j] = p >= 0 && p < j ? p : -1;
        s.token[j] = d;
        if (a.greedy)
            continue;
        s.uniform[j] = a.uniform[base + j];
        if (p >= 0 && p < j && d >= 0 && d < a.V) {
            s.x[j] = to_float(reinterpret_cast<const T *>(row_at<T>(a, b, p, false).p)[d]);
            if (a.draft)
                s.y[j] = to_float(reinterpret_cast<const T *>(row_at<T>(a, b, p, true).p)[d]);
        }
    }
    if constexpr (kWalk) {
        __shared__ WalkShared walked;
        cluster_wait();
        __syncthreads();
        if (a.greedy)
            walk<T, true>(a, s, walked, b, n, cluster, taken, failed);
        else
            walk<T, false>(a, s, walked, b, n, cluster, taken, failed);
    } else {
        pdl_wait();
        __syncthreads();
        if (tid == 0)
            undone = 0;
        static_assert(kMostStreams <= kDraw, "a thread to each CTA's word");
        const uint32_t lost = tid < a.streams ? __ldcg(a.gave_up + tid) : 0;
        sum_rows<T>(a, s, b, n);
        __syncthreads();
        if (lost)
            undone = 1;
        if (a.parents) {
            for (int c = warp; c < n; c += kDraw / 32) {
                const int to = decide(a, s, c, n);
                if (lane == 0)
                    s.choice[c] = (short)to;
            }
        } else {
            for (int c = tid; c < n; c += kDraw)
                s.choice[c] = (short)decide_chain(a, s, c, n);
        }
        __syncthreads();
        if (tid == 0) {
            int at = 0, len = 0;
            for (;; ++len) {
                s.path[len] = (short)at;
                const int to = s.choice[at];
                if (to <= 0) {
                    failed = to == kBad;
                    break;
                }
                at = to;
            }
            taken = len;
        }
    }
    __syncthreads();
    int extra = -1;
    if (!kWalk && (failed || a.greedy))
        cluster_wait();
    if (!failed) {
        const int cur = s.path[taken];
        if (a.greedy) {
            extra = (int)s.first[cur];
        } else {
            if (!a.draft) {
                for (int j = cur + 1 + tid; j < n; j += kDraw) {
                    const int d = s.token[j];
                    if (s.parent[j] == cur && d >= v0 && d < v1)
                        atomicOr(&gone[(d - v0) >> 5], 1u << ((d - v0) & 31));
                }
                __syncthreads();
            }
            const bool rejected = a.draft && cur + 1 < n;
            const T *row = reinterpret_cast<const T *>(row_at<T>(a, b, cur, false).p);
            const T *less = rejected ? reinterpret_cast<const T *>(row_at<T>(a, b, cur, true).p) : row;
            const float pm = s.of[cur].m, pz = 1.0f / s.of[cur].z;
            const float qm = rejected ? s.less[cur].m : 0.0f, qz = rejected ? 1.0f / s.less[cur].z : 0.0f;
            float key = 0.0f;  // the best so far, and its token
            uint32_t at = 0;
            // r / E, where it is more than the best: compared as r > best E, and divided then.  (A NaN or
            // an infinity in E fails the test, what is negative gives no key.)
            auto weigh = [&](float r, float e, int v) {
                if (r > key * e) {
                    const float k = __fdiv_rn(r, e);
                    if (k > key) {
                        key = k;
                        at = v;
                    }
                }
            };
            // of all values of a vector, two at a time; the norm's reciprocal in the exponent
            auto weights = [&](float (&x)[E], uint64_t m2, uint64_t c2, uint64_t l2) {
#pragma unroll
                for (int i = 0; i < E; i += 2) {
                    float t0, t1;
                    un2(fma2(add2(f2(x[i], x[i + 1]), m2), c2, l2), t0, t1);
                    x[i] = ex2_mufu(t0);
                    x[i + 1] = ex2_mufu(t1);
                }
            };
            const float pl = -log2f(s.of[cur].z), ql = rejected ? -log2f(s.less[cur].z) : 0.0f;
            const uint64_t pm2 = f2(-pm, -pm), pc2 = f2(a.ct, a.ct), pl2 = f2(pl, pl);
            const uint64_t qm2 = f2(-qm, -qm), qc2 = f2(a.cd, a.cd), ql2 = f2(ql, ql);
            float bar = 0.0f;
            auto p_of = [&](float x) { return ex2_mufu((x - pm) * a.ct) * pz; };
            auto q_of = [&](float y) { return ex2_mufu((y - qm) * a.cd) * qz; };
            // the largest key, the lowest token where there are several: in warp 0
            auto best_of_warp = [&](uint32_t &k, uint32_t &v) {
                const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, k);
                v = __reduce_min_sync(0xFFFFFFFFu, k == top ? v : kNoIdx);
                k = top;
            };
            auto best_of_cta = [&]() -> unsigned long long {
                uint32_t k = __float_as_uint(key), v = at;
                best_of_warp(k, v);
                if (lane == 0)
                    best[warp] = make_uint2(k, v);
                __syncthreads();
                if (warp == 0) {
                    const uint2 o = lane < kDraw / 32 ? best[lane] : make_uint2(0, kNoIdx);
                    k = o.x;
                    v = o.y;
                    best_of_warp(k, v);
                }
                return k ? ((unsigned long long)k << 32) | (0xFFFFFFFFu - v) : 0;
            };
            if (((reinterpret_cast<uintptr_t>(row) | reinterpret_cast<uintptr_t>(less) |
                  reinterpret_cast<uintptr_t>(noise)) & 15u) == 0 && a.V % E == 0) {
                constexpr int kTwo = 2;  // vectors of a thread in flight
                for (int w0 = v0 + warp * 32 * E; w0 < v1; w0 += kTwo * kDraw * E) {
                    const int w = w0 + lane * E;
                    uint4 xr[kTwo], yr[kTwo];
                    float4 er[kTwo][E / 4];
#pragma unroll
                    for (int k = 0; k < kTwo; ++k) {
                        const int v = w + k * kDraw * E;
                        if (v >= v1)
                            continue;
                        xr[k] = *reinterpret_cast<const uint4 *>(row + v);
                        if (rejected)
                            yr[k] = *reinterpret_cast<const uint4 *>(less + v);
#pragma unroll
                        for (int i = 0; i < E / 4; ++i)
                            er[k][i] = reinterpret_cast<const float4 *>(noise + v)[i];
                    }
#pragma unroll
                    for (int k = 0; k < kTwo; ++k) {
                        const int v = w + k * kDraw * E;
                        if (v >= v1)
                            continue;
                        float x[E], y[E];
                        widen<T>(xr[k], x);
                        weights(x, pm2, pc2, pl2);
                        if (rejected) {
                            widen<T>(yr[k], y);
                            weights(y, qm2, qc2, ql2);
#pragma unroll
                            for (int i = 0; i < E; ++i)
                                x[i] -= y[i];
                        }
                        const uint32_t out = gone[(v - v0) >> 5] >> ((v - v0) & 31);
                        if (out & ((1u << E) - 1))
#pragma unroll
                            for (int i = 0; i < E; ++i)
                                x[i] = (out >> i) & 1u ? 0.0f : x[i];
                        // whether one of them is more than the warp's best
                        float most = -1.0f;
#pragma unroll
                        for (int i = 0; i < E / 4; ++i) {
                            const float4 f = er[k][i];
                            most = max3(most, fmaf(-bar, f.x, x[4 * i]), fmaf(-bar, f.y, x[4 * i + 1]));
                            most = max3(most, fmaf(-bar, f.z, x[4 * i + 2]), fmaf(-bar, f.w, x[4 * i + 3]));
                        }
                        if (most > 0.0f)
#pragma unroll
                            for (int i = 0; i < E; ++i) {
                                const float4 f = er[k][i / 4];
                                weigh(x[i], i % 4 == 0 ? f.x : i % 4 == 1 ? f.y : i % 4 == 2 ? f.z : f.w, v + i);
                            }
                    }
                    bar = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(key)));
                }
            } else {
                constexpr int kMany = 8;  // values of a thread in flight
                for (int w = v0 + tid; w < v1; w += kMany * kDraw) {
                    T x[kMany], y[kMany];
                    float e[kMany];
#pragma unroll
                    for (int k = 0; k < kMany; ++k) {
                        const int v = min(w + k * kDraw, v1 - 1);
                        x[k] = row[v];
                        y[k] = less[v];
                        e[k] = noise[v];
                    }
#pragma unroll
                    for (int k = 0; k < kMany; ++k) {
                        const int v = w + k * kDraw;
                        if (v >= v1)
                            break;
                        float r = p_of(to_float(x[k]));
                        if (rejected)
                            r -= q_of(to_float(y[k]));
                        weigh((gone[(v - v0) >> 5] >> ((v - v0) & 31)) & 1u ? 0.0f : r, e[k], v);
                    }
                }
            }
            unsigned long long top = best_of_cta();
            if (!kWalk)
                cluster_wait();
            if (tid == 0)
                cluster.map_shared_rank(of_cta, 0)[rank] = top;
            cluster_arrive();
            if (rank != 0)
                return;
            cluster_wait();
            top = of_cta[0];
            for (int i = 1; i < ranks; ++i)
                top = of_cta[i] > top ? of_cta[i] : top;
            // no weight left: from p itself, and then its largest, by this CTA alone
            for (int turn = 1; turn < 3 && top == 0; ++turn) {
                for (int v = tid; v < a.V; v += kDraw)
                    weigh(p_of(to_float(row[v])), turn == 1 ? noise[v] : 1.0f, v);
                top = best_of_cta();
                __syncthreads();
                if (tid == 0)
                    of_cta[0] = top;
                __syncthreads();
                top = of_cta[0];
            }
            extra = (int)(0xFFFFFFFFu - (uint32_t)top);
        }
    }
    if (rank != 0)
        return;
    const bool dead = (!kWalk && undone) || (__ldcg(a.status) & kDevStatTimeout) != 0;
    for (int j = tid; j < a.M; j += kDraw) {
        int token = -1, node = -1;
        if (!failed && !dead && j <= taken) {
            node = s.path[j];
            token = j < taken ? s.token[s.path[j + 1]] : extra;
        }
        a.out_tokens[base + j] = token;
        a.out_nodes[base + j] = node;
    }
    if (tid == 0)
        a.out_n[b] = dead ? FDLLM_ROW_DEVICE_ERROR : failed ? FDLLM_ROW_NONFINITE : taken;
}

// Whether rows are read as the walk comes to them.
bool walks(const VerifyArgs &a, int es)
{
    const int64_t row = (int64_t)a.V * es;
    return a.parents && a.B * (a.M * row) >= (row > kSmallRow ? kWalkLong : kWalkShort);
}

// CTAs that share a sequence's rows then: a cluster of as many for each sequence at once, where there is
// room.
// `held`: the clusters of 1, 2, 4 and 8 that the GPU holds.
int walk_ranks(const VerifyArgs &a, int es, const std::atomic<int> *held)
{
    int i = 0;
    while (i < 3 && a.B <= held[i + 1] && (int64_t)a.V * es >> i > kWalkShare)
        ++i;
    return 1 << i;
}

// CTAs that share a sequence's draw: as many as fill the GPU once (two to an SM), where a slice keeps
// four values or so of a thread; and as many as a slice's bits of taken tokens need.
int draw_ranks(const VerifyArgs &a)
{
    if (a.greedy)
        return 1;
    int ranks = 1;
    while (ranks < kMaxRanks && ((int64_t)a.B * ranks * 2 <= 2 * sm_count() || a.V / ranks > (1 << 17)) &&
           a.V / ranks >= 4096)
        ranks *= 2;
    return ranks;
}

template <typename T>
cudaError_t launch_verify(const VerifyArgs &a, cudaStream_t s)
{
    constexpr int kMostDraw = kMaxNodes * Nodes::kBytes + kMaxRowV / 8;
    static PerDevice ready;
    static std::atomic<int> held[kMaxCacheDevices][4];
    cudaError_t e = ready.once([] {
        cudaFuncAttributes f;  // (asked for, a kernel is loaded: a capture may be next)
        cudaError_t r = cudaFuncGetAttributes(&f, verify_small_kernel<T, true>);
        if (r == cudaSuccess)
            r = cudaFuncGetAttributes(&f, verify_small_kernel<T, false>);
        if (r == cudaSuccess)
            r = cudaFuncSetAttribute(verify_stream_kernel<T, true>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem);
        if (r == cudaSuccess)
            r = cudaFuncSetAttribute(verify_stream_kernel<T, false>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem);
        if (r == cudaSuccess)
            r = cudaFuncSetAttribute(verify_draw_kernel<T, false>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, kMostDraw);
        if (r == cudaSuccess)
            r = cudaFuncSetAttribute(verify_draw_kernel<T, true>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, kMostDraw);
        int dev = 0;
        if (r == cudaSuccess && (r = cudaGetDevice(&dev)) == cudaSuccess)
            for (int i = 0; i < 4; ++i)
                held[dev][i] = clusters_held(verify_draw_kernel<T, true>, kDraw, kMostDraw, 1 << i);
        return r;
    });
    if (e != cudaSuccess)
        return e;
    const int64_t rows = (int64_t)a.B * (a.draft ? 2 * a.M - 1 : a.M);
    auto small = a.greedy ? verify_small_kernel<T, true> : verify_small_kernel<T, false>;
    auto stream = a.greedy ? verify_stream_kernel<T, true> : verify_stream_kernel<T, false>;
    VerifyArgs call = a;
    int walkers = 0;
    if (walks(a, sizeof(T))) {
        int dev = 0;
        if ((e = cudaGetDevice(&dev)) != cudaSuccess)
            return e;
        walkers = walk_ranks(a, sizeof(T), held[dev]);
    }
    if (walkers == 0 && (int64_t)a.V * sizeof(T) <= kSmallRow) {
        const int64_t want = (rows * a.per + 7) / 8, most = (int64_t)sm_count() * 8;
        e = launch(small, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, s, true, a);
    } else if (walkers == 0) {
        const int64_t units = rows * a.pieces, most = sm_count() < kMostStreams ? sm_count() : kMostStreams;
        call.streams = (int)(units < most ? units : most);
        e = launch(stream, dim3((unsigned)call.streams), dim3(kMath + 32), kStreamSmem, s, true, call);
    }
    if (e != cudaSuccess)
        return e;
    const int ranks = walkers != 0 ? walkers : draw_ranks(a);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.B * ranks));
    cfg.blockDim = dim3(kDraw);
    cfg.dynamicSmemBytes = draw_smem(a.M, a.V, ranks, a.greedy);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)ranks, 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = plain_launches ? 1 : 2;
    if (walkers == 0)
        return cudaLaunchKernelEx(&cfg, verify_draw_kernel<T, false>, call);
    const int64_t share = (int64_t)a.V * (int)sizeof(T) / ranks;
    auto rows_of = [&](int64_t bytes) {
        return (int)(bytes < share ? 1 : bytes / share < kTurn ? bytes / share : kTurn);
    };
    call.turn = rows_of(kTurnBytes);
    call.turn_most = rows_of(2 * kTurnBytes);
    return cudaLaunchKernelEx(&cfg, verify_draw_kernel<T, true>, call);
}

// How rows are cut: whole, or in pieces of whole chunks so that every SM has two, and no piece is
// longer than four chunks (where rows are many, pieces of one, two and four are alike within 2 %).  The SMs
// are counted as 152: the workspace's size goes by it, and that asks no GPU.  With one piece to an SM,
// rows in the L2: 16 greedy chains of 17 of 50021 fp32 values 11.5 us for 13.0, 16 chains of nine of 126464
// 22.8 for 25.4; with four 13.2 and 24.0; fewer rows are alike.
void cut_rows(int64_t rows, int V, int es, int &pieces, int &piece_vecs, int &per)
{
    if ((int64_t)V * es <= kSmallRow) {
        pieces = per = 1;
        piece_vecs = 0;
        while (per < 8 && (int64_t)V * es / 16 > per * 32 * kSmallVecs)
            per *= 2;
        return;
    }
    // vectors that a row has wherever it begins, so that no piece is empty
    const int E = 16 / es, vecs = (V - (E - 1)) / E;
    const int chunks = (vecs + kChunkVecs - 1) / kChunkVecs;
    int of = 4;
    while (of > 1 && rows * ((chunks + of - 1) / of) < 2 * 152)
        --of;
    pieces = (chunks + of - 1) / of;
    piece_vecs = of * kChunkVecs;
    per = pieces * kMathWarps;
}

int64_t verify_rows(int B, int M) { return (int64_t)B * (2 * (int64_t)M - 1); }

size_t verify_bytes(int B, int M, int V, int dtype)
{
    int pieces, vecs, most = 0;
    // (with the draft's rows or without)
    for (int64_t rows : {verify_rows(B, M), (int64_t)B * M}) {
        int per;
        cut_rows(rows, V, rows_esize(dtype), pieces, vecs, per);
        most = per > most ? per : most;
    }
    return kMostStreams * 4 + ((size_t)verify_rows(B, M) * most * sizeof(UnitPartial) + 255) / 256 * 256;
}

bool verify_sizes(int B, int M, int V)
{
    // (pieces are counted in 32 bits)
    return B >= 1 && B <= kMaxGridYZ && M >= 1 && M <= kMaxNodes && V >= 1 && V <= kMaxRowV &&
           verify_rows(B, M) * (V / 4096 + 1) < ((int64_t)1 << 31);
}

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" {

size_t fdllm_verify_draft_workspace_bytes(int B, int M, int V, int dtype)
{
    return verify_sizes(B, M, V) && rows_dtype(dtype) ? verify_bytes(B, M, V, dtype) : 0;
}

fdllm_status fdllm_verify_draft(const void *target, const int64_t *target_strides,
                                const void *draft, const int64_t *draft_strides, int dtype, int B,
                                int M, int V, const int32_t *tokens, const int32_t *parents,
                                const int32_t *lens, double temperature, double draft_temperature,
                                const float *uniform, const float *noise, int32_t *out_tokens,
                                int32_t *out_nodes, int32_t *out_n, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    const bool greedy = temperature == 0.0;
    auto sane = [](double t) { return t >= 1e-6 && t <= 1e6; };
    if (!verify_sizes(B, M, V) || !rows_dtype(dtype) || !target || !target_strides ||
        (draft && !draft_strides) || !tokens || !out_tokens ||
        !out_nodes || !out_n || (!greedy && (!sane(temperature) || !uniform || !noise)) ||
        (draft && (greedy || parents || !sane(draft_temperature))))
        return FDLLM_ERR_ARG;
    if (((reinterpret_cast<uintptr_t>(target) | reinterpret_cast<uintptr_t>(draft)) &
         (uintptr_t)(rows_esize(dtype) - 1)) != 0)
        return FDLLM_ERR_ALIGN;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
        workspace_bytes < verify_bytes(B, M, V, dtype))
        return FDLLM_ERR_WORKSPACE;
    VerifyArgs a = {};
    a.target = target;
    a.draft = M > 1 ? draft : nullptr;
    a.t_batch = target_strides[0];
    a.t_row = target_strides[1];
    if (a.draft) {
        a.d_batch = draft_strides[0];
        a.d_row = draft_strides[1];
    }
    a.B = B;
    a.M = M;
    a.V = V;
    a.tokens = tokens;
    a.parents = parents;
    a.lens = lens;
    a.greedy = greedy;
    a.ct = (float)(1.4426950408889634 / (greedy ? 1.0 : temperature));
    a.cd = a.draft ? (float)(1.4426950408889634 / draft_temperature) : a.ct;
    a.uniform = uniform;
    a.noise = noise;
    a.out_tokens = out_tokens;
    a.out_nodes = out_nodes;
    a.out_n = out_n;
    a.gave_up = static_cast<uint32_t *>(workspace);
    a.parts = reinterpret_cast<UnitPartial *>(a.gave_up + kMostStreams);
    cut_rows((int64_t)B * (a.draft ? 2 * M - 1 : M), V, rows_esize(dtype), a.pieces, a.piece_vecs, a.per);
    a.status = cache_status_word();
    if (!a.status)
        return FDLLM_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == FDLLM_BF16   ? launch_verify<__nv_bfloat16>(a, s)
                          : dtype == FDLLM_FP16 ? launch_verify<__half>(a, s)
                                                : launch_verify<float>(a, s);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

}  // extern "C"
