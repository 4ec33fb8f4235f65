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
constexpr int kThreads = 128;      // of a CTA of the small form
// Rows up to kSmallRow bytes take it, and up to kManyRow where there are more rows than SMs: each
// further row of a CTA costs the long form about 5 us whatever its length, for the latencies from list
// to mark, which many CTAs to an SM hide.  Steps in bf16: 1024 rows of 12001 13 us (the long form 34), 256
// of 17000 8.7 (15), 4096 of 32000 116 (150), 300 of 32000 12.2 (15.4; half of them masked 12.3, 11.0); but
// 64 of 32000 10.2 (9.5), 1024 of 45000, half of them masked, 36 (34), 2048 of 64000 131 (113): their
// second read is no longer the L2's.  The loss alone has none, and rows of up to kLossV values take it
// where there are more than kFull to an SM: 2056 of 50021 in fp32, 0.6 of them masked, 43 us (49), 4096
// of 126464, half of them masked, 86 (95); but 256 of 126464 32 (19).
constexpr int kSmallRow = 32768, kManyRow = 65536;
constexpr int kLossV = 1 << 17, kFull = 8;

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
    uint32_t *status;        // sticky: a bounded wait gave up
};

__device__ __forceinline__ float top_value(const DistillArgs &a, int64_t i)
{
    if (a.top_dtype == FDLLM_FP32)
        return static_cast<const float *>(a.top)[i];
    if (a.top_dtype == FDLLM_BF16)
        return __bfloat162float(static_cast<const __nv_bfloat16 *>(a.top)[i]);
    return __half2float(static_cast<const __half *>(a.top)[i]);
}

// A listed token's weight is e^(t / T - lse), t the teacher's logit, or e^((t - most) / T) relative to the
// list's largest.  There the difference comes first, as with the student's logits: of logits within a
// factor of two it is exact, where t / T, rounded by itself, is off by 2^-24 of its size (logits near 8
// at T = 1e-3: 5e-4 of the weight); times 1 / T, it is off by 2^-23 of the exponent.  Against a given lse
// the quotient is as exact as lse itself is.
__device__ __forceinline__ float score(const DistillArgs &a, float t)
{
    return a.lse ? __fdiv_rn(t, a.temperature) : t;
}
__device__ __forceinline__ float exponent(const DistillArgs &a, float score, float most_or_lse)
{
    const float d = score - most_or_lse;
    return a.lse ? d : d * a.inv_t;
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

// -inf in the place of the values whose bits are set.
template <typename T>
__device__ __forceinline__ void leave_out(uint4 &r, uint32_t bits)
{
    constexpr uint32_t kPad = no_values<T>();
    uint32_t *w = reinterpret_cast<uint32_t *>(&r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = (bits >> i) & 1u ? kPad : w[i];
        } else {
            const uint32_t keep = ((bits >> (2 * i)) & 1u ? 0u : 0xFFFFu) |
                                  ((bits >> (2 * i + 1)) & 1u ? 0u : 0xFFFF0000u);
            w[i] = (w[i] & keep) | (kPad & ~keep);
        }
    }
}

// f 2^((x - m) c) of a vector's values: as Summed's terms are taken, what the rounding of m c leaves in f.
struct RowTerms {
    uint64_t f2f, c2, n2;
    bool far;
    __device__ __forceinline__ RowTerms(float m, float c, float f)
    {
        const float ref = m * c;
        far = !(fabsf(ref) < kFar);
        if (!far)
            f *= ex2_mufu(-fmaf(m, c, -ref));
        f2f = f2(f, f);
        c2 = f2(c, c);
        n2 = far ? f2(-m, -m) : f2(-ref, -ref);
    }
    template <typename T>
    __device__ __forceinline__ uint4 of(const uint4 &x) const
    {
        constexpr int E = 16 / sizeof(T);
        float y[E];
        widen<T>(x, y);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const uint64_t y2 = f2(y[e], y[e + 1]);
            float t0, t1;
            un2(far ? mul2(add2(y2, n2), c2) : fma2(y2, c2, n2), t0, t1);
            un2(mul2(f2(ex2_mufu(t0), ex2_mufu(t1)), f2f), y[e], y[e + 1]);
        }
        return narrow<T>(y);
    }
};

// ---- Short rows: a CTA of kThreads to a row, many on an SM.
// kSum: the row's sums are taken (else they are given); kGrad: the gradient is written; kMine: listed
// tokens of a thread.
// The sum alone of fp32 rows: nine CTAs to an SM (1234 rows of 50021 43.6 us, with eight 52.6: more rows than
// those hold at once).  In 16 bits eight and 64 registers: 2048 rows of 126464 85.6 us, with nine 89.3.
template <typename T, bool kSum, bool kGrad, int kMine>
constexpr int small_ctas()
{
    return kSum && !kGrad && kMine == 1 && sizeof(T) == 4 ? kFull + 1 : kFull;
}
template <typename T, bool kSum, bool kGrad, int kMine>
__global__ void __launch_bounds__(kThreads, small_ctas<T, kSum, kGrad, kMine>())
    distill_small_kernel(const __grid_constant__ DistillArgs a)
{
    constexpr int E = 16 / sizeof(T);
    constexpr int kWarps = kThreads / 32;
    constexpr int kFour = kGrad ? 4 : 8;  // vectors of a thread in flight
    extern __shared__ __align__(16) uint32_t marks[];  // a bit for each value of the whole vectors
    __shared__ int idx[kMine * kThreads];
    __shared__ float p[kMine * kThreads];
    __shared__ float of_most[kWarps], of_mass[kWarps];
    __shared__ ExpSum of_rest[kWarps], of_listed[kWarps];
    __shared__ float of_loss[kWarps], of_share[kWarps];
    __shared__ uint32_t ends;  // of the values before the whole vectors (8 bits), and behind
    __shared__ int twice;
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const float c = a.inv_t * kLog2e;
    const uint8_t *const listed = reinterpret_cast<const uint8_t *>(marks);
    bool clean = false;
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
        if (!clean)
            for (int i = tid; i < a.V / 32 + 1; i += kThreads)
                marks[i] = 0;
        clean = true;
        if (tid == 0)
            twice = 0, ends = 0;
        __syncthreads();
        int v[kMine];
        float m[kMine], x[kMine];
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
                    m[j] = score(a, top_value(a, row * a.K + k));
                    x[j] = to_float(s.row[at]);
                }
                idx[k] = v[j];
                most = Most()(most, m[j]);
            }
        }
        // its marks
#pragma unroll
        for (int j = 0; j < kMine; ++j)
            if (v[j] >= 0) {
                const int b = v[j] - s.head;
                const bool end = v[j] < s.head || v[j] >= s.tail();
                const int bit = v[j] < s.head ? v[j] : end ? 8 + v[j] - s.tail() : b & 31;
                if ((atomicOr(end ? &ends : &marks[b >> 5], 1u << bit) >> bit) & 1u)
                    twice = 1;
            }
        if (!a.lse) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                most = Most()(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
            if (lane == 0)
                of_most[warp] = most;
        }
        __syncthreads();
        if (a.lse) {
            most = a.lse[row];
        } else {
            most = of_most[0];
            for (int w = 1; w < kWarps; ++w)
                most = Most()(most, of_most[w]);
        }
        float P = 0.0f, R = 0.0f;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            m[j] = v[j] >= 0 ? expf(exponent(a, m[j], most)) : 0.0f;
            P += m[j];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            P += __shfl_xor_sync(0xFFFFFFFFu, P, o);
        if (lane == 0)
            of_mass[warp] = P;
        __syncthreads();
        P = of_mass[0];
        for (int w = 1; w < kWarps; ++w)
            P += of_mass[w];
        if (a.lse) {
            if (kSum)
                P = most == most ? P : most;  // (a NaN, also where nothing is listed)
            R = fmaxf(1.0f - P, 0.0f);
        } else if (P != 0.0f) {
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (m[j] != 0.0f)
                    m[j] = __fdiv_rn(m[j], P);
            P = P == P ? 1.0f : P;
        }
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
        const int end = lane < 8 ? lane : s.tail() + lane - 8;  // warp 0: a value of the ends
        const bool has_end = warp == 0 && lane < 16 && (lane < 8 ? end < s.head : end < a.V);
        float M, Z;
        ExpSum rest;
        if (kSum) {
            // ---- the tokens that are not listed
            Summed sum;
            for (int i0 = tid; i0 < s.vecs; i0 += kFour * kThreads) {
                constexpr uint32_t kPad = no_values<T>();
                uint4 y[kFour];
#pragma unroll
                for (int q = 0; q < kFour; ++q) {
                    const int i = i0 + q * kThreads;
                    y[q] = i < s.vecs ? s.vectors()[i] : make_uint4(kPad, kPad, kPad, kPad);
                }
#pragma unroll
                for (int q = 0; q < kFour; ++q) {
                    const int i = i0 + q * kThreads;
                    const uint32_t bits = i >= s.vecs ? 0u
                                          : E == 8    ? listed[i]
                                                      : (listed[i >> 1] >> (4 * (i & 1))) & 15u;
                    if (bits)
                        leave_out<T>(y[q], bits);
                }
                sum.add<T, kFour>(y, c);
            }
            sum.settle(c);
            if (has_end && !((ends >> lane) & 1u))
                sum.z.add(to_float(s.row[end]), c);
            __syncwarp();
            // ---- and the listed ones: each warp's, relative to their own maximum
            ExpSum of_x;
            float A = 0.0f, share = 0.0f;
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (v[j] >= 0)
                    of_x.m = Most()(of_x.m, x[j]);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                of_x.m = Most()(of_x.m, __shfl_xor_sync(0xFFFFFFFFu, of_x.m, o));
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (v[j] >= 0) {
                    of_x.z += ex2_mufu((x[j] - of_x.m) * c);
                    if (m[j] != 0.0f)
                        A += m[j] * (logf(m[j]) - (x[j] - of_x.m) * a.inv_t);
                    share += m[j];
                }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                of_x.z += __shfl_xor_sync(0xFFFFFFFFu, of_x.z, o);
                A += __shfl_xor_sync(0xFFFFFFFFu, A, o);
                share += __shfl_xor_sync(0xFFFFFFFFu, share, o);
            }
            rest = warp_sum(sum.z, c);
            if (lane == 0) {
                of_rest[warp] = rest;
                of_listed[warp] = of_x;
                of_loss[warp] = A;
                of_share[warp] = share;
            }
            __syncthreads();
            rest = of_rest[0];
            M = of_listed[0].m;
            for (int w = 1; w < kWarps; ++w) {
                rest.merge(of_rest[w], c);
                M = Most()(M, of_listed[w].m);
            }
            M = Most()(M, rest.m);
            Z = rest.z * ex2_mufu((rest.m - M) * c);
            for (int w = 0; w < kWarps; ++w)
                Z += of_listed[w].z * ex2_mufu((of_listed[w].m - M) * c);
            if (!(Z > 0.0f && Z <= FLT_MAX) || !finite_f(M) || P != P)
                Z = nan_f();  // (and all that is made of it)
            if (rest.z == 0.0f)
                R = 0.0f;
            if (tid == 0) {
                const float log_z = logf(Z);
                float loss = 0.0f;
                for (int w = 0; w < kWarps; ++w) {
                    loss += of_loss[w];
                    if (of_share[w] != 0.0f)
                        loss += of_share[w] * ((M - of_listed[w].m) * a.inv_t + log_z);
                }
                if (R > 0.0f)
                    loss += R * (logf(R) - ((rest.m - M) * a.inv_t + logf(rest.z) - log_z));
                a.loss[row] = Z == Z ? loss : Z;
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
            const float r = rest.z * ex2_mufu((rest.m - M) * c) / Z;
            // of s_v relative to the reference of the others
            float f = rest.z == 0.0f ? (Z == Z ? 0.0f : Z) : scale * (r * (P + R) - R) / rest.z;
            if (has_end)
                grad[end] = from_float<T>(ex2_mufu((to_float(s.row[end]) - rest.m) * c) * f);
            const RowTerms terms(rest.m, c, f);
            uint4 *out = reinterpret_cast<uint4 *>(grad + s.head);
            for (int i0 = tid; i0 < s.vecs; i0 += kFour * kThreads) {
                uint4 y[kFour];
#pragma unroll
                for (int q = 0; q < kFour; ++q)
                    if (i0 + q * kThreads < s.vecs)
                        y[q] = s.vectors()[i0 + q * kThreads];
#pragma unroll
                for (int q = 0; q < kFour; ++q)
                    if (i0 + q * kThreads < s.vecs)
                        __stcs(out + i0 + q * kThreads, terms.template of<T>(y[q]));
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (v[j] >= 0)
                    grad[v[j]] = from_float<T>(
                        scale * (ex2_mufu((x[j] - M) * c) / Z * (P + R) - m[j]));
        } else {
            __syncthreads();
        }
        // (the marks of a token's other places go with its first)
        for (int k = tid; k < a.K; k += kThreads)
            if (idx[k] >= s.head && idx[k] < s.tail())
                marks[(idx[k] - s.head) >> 5] = 0;
    }
}

// ---- Longer rows: a CTA, or a cluster of them, holds a row in shared memory from its sum to its
// gradient.
//
// Roles.  Sixteen warps walk the row (the sum, then the gradient); eight look after the teacher: for the
// row to come they read its list and the student's logits of it, make the probabilities and what
// else is of the list alone, and mark the listed tokens, and for the row before they write the
// listed tokens' gradients over what the sixteen wrote there; one lane copies rows into a ring of
// shared memory, and one warp writes the rows of zeros.
//
// The ring.  Chunks of a row come in order; the first pass gives back those that the ring cannot
// hold beside the others, which come again (from the L2, where they have just been) behind the
// row's last; the second pass starts with the oldest that is still there, and each chunk it gives back
// makes room for one of the next row.
constexpr int kMathWarps = 16, kMath = 32 * kMathWarps;
constexpr int kTeachers = 256;
constexpr int kRingThreads = kMath + kTeachers + 64;
constexpr int kChunk = 32768, kChunkVecs = kChunk / 16, kPer = kChunkVecs / kMath;
constexpr int kMostListed = 1 << 17;  // tokens of a CTA's share of a row: their bits take 16 KB
constexpr int kMarks = kMostListed / 8 + 32;
constexpr int kZeros = 2048;
constexpr int kMaxRanks = 8;
enum { kBarMath = 1, kBarTeach };

// The masked rows, or the others, of this cluster: every n-th of them.  A warp looks at 512 rows at a
// time, 16 to a lane.
struct RowWalk {
    const uint8_t *mask;
    int64_t rows, base, before;  // rows below base are passed, `before` of the kind among them
    uint32_t bits, upto;         // this lane's 16 rows; how many of the kind up to and with them
    int in_block;
    bool masked;

    __device__ __forceinline__ void load()
    {
        const int64_t r = base + 16 * (threadIdx.x & 31);
        bits = 0;
        if (r + 16 <= rows && (reinterpret_cast<uintptr_t>(mask + r) & 15u) == 0) {
            const uint4 v = *reinterpret_cast<const uint4 *>(mask + r);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 16; ++i)
                bits |= ((w[i >> 2] >> (8 * (i & 3))) & 0xFFu) != 0 ? 1u << i : 0u;
        } else {
            for (int i = 0; i < 16 && r + i < rows; ++i)
                bits |= mask[r + i] != 0 ? 1u << i : 0u;
        }
        if (!masked)
            bits = ~bits & (r >= rows ? 0u : r + 16 <= rows ? 0xFFFFu : (1u << (rows - r)) - 1);
        upto = __popc(bits);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            upto += (threadIdx.x & 31) >= o ? x : 0;
        }
        in_block = (int)__shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    __device__ __forceinline__ RowWalk(const uint8_t *m, int64_t n, bool of_masked)
        : mask(m), rows(n), base(0), before(0), masked(of_masked)
    {
        load();
    }
    // The rank-th row of the kind (ranks grow from call to call), -1: there are not so many.
    __device__ __forceinline__ int64_t find(int64_t rank)
    {
        while (rank >= before + in_block) {
            if (base + 512 >= rows)
                return -1;
            before += in_block;
            base += 512;
            load();
        }
        const uint32_t in = (uint32_t)(rank - before);
        const uint32_t lane = __ffs(__ballot_sync(0xFFFFFFFFu, upto > in)) - 1;
        uint32_t skip = in - (upto - __popc(bits)), b = bits;
        if ((threadIdx.x & 31) == lane)
            for (; skip > 0; --skip)
                b &= b - 1;
        const int at = __shfl_sync(0xFFFFFFFFu, __ffs(b) - 1, lane);
        return base + 16 * lane + at;
    }
};

// A CTA's share of a row: whole vectors [v0, v1), the first CTA's with the values before them, the
// last's with those behind.
template <typename T>
struct RowShare {
    RowSpan<T> r;
    int v0, v1;
    __device__ __forceinline__ RowShare(const void *base, int64_t row, int V, int rank, int ranks)
        : r(static_cast<const T *>(base) + row * V, V)
    {
        const int per = (r.vecs + ranks - 1) / ranks;
        v0 = min(r.vecs, rank * per);
        v1 = min(r.vecs, v0 + per);
    }
    // Whether value v of the row is the CTA's.
    __device__ __forceinline__ bool holds(int v, int rank, int ranks) const
    {
        constexpr int E = RowSpan<T>::E;
        const int b = v - r.head;
        return v < r.head ? rank == 0 : v >= r.tail() ? rank == ranks - 1 : b >= v0 * E && b < v1 * E;
    }
    __device__ __forceinline__ int chunks() const { return (v1 - v0 + kChunkVecs - 1) / kChunkVecs; }
    __device__ __forceinline__ int in_chunk(int j) const { return min(kChunkVecs, v1 - v0 - j * kChunkVecs); }
};

// What the teachers' warps leave for a row.
struct Taught {
    int64_t row;         // -1: no more
    float P, R;
    float A;             // sum p_k (log p_k - (x_k - m) / T)
    ExpSum x;            // of the listed tokens' logits
    float scale;         // gradient of the loss / T
    uint32_t ends;       // a bit for each listed value out of the whole vectors: 8 before, 8 behind
    float M, Z;          // of all tokens, and
    ExpSum rest;         // of the others, where they are given
};

struct RingShared {
    uint64_t full[6], empty[6];
    uint64_t ready[2];    // of a row, by parity: its list is taught
    uint64_t swept[2];    // the first pass is done, its marks are not needed
    uint64_t written[2];  // the second is done, the listed tokens may be written
    uint64_t crossed[2];  // the cluster's sums are here
    Taught taught[2];
    float4 fix[2];        // for the listed tokens: M, Z, P + R, scale
    ExpSum part[2][kMathWarps];
    ExpSum of_rank[2][kMaxRanks];
    float reduce[3][kTeachers / 32];
    uint32_t groups[2][kMostListed / 4 / 1024];  // a bit for each 32 vectors that hold a marked value
    int twice;
    uint32_t ends;
};

// Shared memory.  With two sets of marks the row to come is marked while the row before is still under
// way (with one, 1234 rows of 50021 logits in fp32 took 64 us, not 53).  The sum alone holds no row
// back and has room for them with a stage less; beside the gradient a set is half as long, and there
// are two where a share fits that.
template <bool kSum, bool kGrad>
struct RingLayout {
    static constexpr bool wide = kSum && !kGrad;
    static constexpr int stages = wide ? 5 : 6;
    static constexpr int set = wide ? kMarks : kMarks / 2;  // bytes of one of two sets
    static constexpr int listed = stages * kChunk, zeros = listed + (wide ? 2 : 1) * kMarks;
    static constexpr int dup = zeros + kZeros, shared = dup + kMaxTop * 8;
    static constexpr int bytes = shared + (int)sizeof(RingShared);
    static_assert(bytes <= 227 * 1024 && shared % 16 == 0 && zeros % 16 == 0, "shared memory");
};

// Eight bytes to another CTA of the cluster, counted by a barrier there.
__device__ __forceinline__ void send_sum(const ExpSum *slot, const uint64_t *bar, int to, const ExpSum &v)
{
    uint32_t at, b;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_addr(slot)), "r"(to));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(smem_addr(bar)), "r"(to));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(at),
                 "r"(__float_as_uint(v.m)), "r"(__float_as_uint(v.z)), "r"(b)
                 : "memory");
}

// This thread's vectors of a chunk of n; `pad` in the words of those that are not there.
template <typename T>
__device__ __forceinline__ void load_chunk(uint4 (&x)[kPer], const uint4 *buf, int n, uint32_t pad)
{
    if (n == kChunkVecs) {
#pragma unroll
        for (int q = 0; q < kPer; ++q)
            x[q] = buf[threadIdx.x + q * kMath];
    } else {
#pragma unroll
        for (int q = 0; q < kPer; ++q) {
            const int v = threadIdx.x + q * kMath;
            x[q] = v < n ? buf[v] : make_uint4(pad, pad, pad, pad);
        }
    }
}

// Sum (or maximum) over the teachers' warps, the same bits in every thread.
template <typename F>
__device__ __forceinline__ float teach_reduce(float x, float *of_warp, F f)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        x = f(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    if ((threadIdx.x & 31) == 0)
        of_warp[(threadIdx.x - kMath) >> 5] = x;
    named_sync(kBarTeach, kTeachers);
    x = of_warp[0];
#pragma unroll
    for (int i = 1; i < kTeachers / 32; ++i)
        x = f(x, of_warp[i]);
    return x;
}

template <typename T, bool kSum, bool kGrad>
__global__ void __launch_bounds__(kRingThreads, 1)
    distill_ring_kernel(const __grid_constant__ DistillArgs a, int ranks, int two)
{
    constexpr int E = 16 / sizeof(T);
    using Layout = RingLayout<kSum, kGrad>;
    constexpr int kStages = Layout::stages;
    extern __shared__ __align__(128) uint8_t smem[];
    // a bit for each value of the share's vectors; with two sets, by the row's parity
    uint8_t *const marks = smem + Layout::listed;
    RingShared &sm = *reinterpret_cast<RingShared *>(smem + Layout::shared);
    const int tid = threadIdx.x, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), lane = tid & 31;
    const int rank = blockIdx.x % ranks, cluster = blockIdx.x / ranks, clusters = gridDim.x / ranks;
    const float c = a.inv_t * kLog2e;
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], kMathWarps);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.ready[i], 1);
            mbar_init(&sm.swept[i], 1);
            mbar_init(&sm.written[i], kMathWarps);
            mbar_init(&sm.crossed[i], 1);
        }
        fence_mbar_init();
    }
    for (int i = tid; i < (Layout::zeros - Layout::listed + kZeros) / 4; i += kRingThreads)
        reinterpret_cast<uint32_t *>(marks)[i] = 0;
    fence_async_smem();
    __syncthreads();
    if (ranks > 1) {
        cluster_arrive();
        cluster_wait();
    }
    pdl_wait();
    // A wait that gave up: no further wait.  Math's and the teachers' warps leave by a vote, before
    // they look at what was never left for them.
    bool dead = false;
    auto wait = [&](uint64_t *bar, uint32_t parity) {
        if (!dead && !mbar_wait(bar, parity, a.status))
            dead = true;
    };

    if (warp < kMathWarps) {
        // ------------------------------------------------------------ the row
        uint32_t kb = 0;  // chunks of the rows before
        for (uint32_t i = 0;; ++i) {
            const uint32_t par = i & 1;
            wait(&sm.ready[par], (i >> 1) & 1);
            const Taught &of = sm.taught[par];
            if (named_sync_or(kBarMath, kMath, dead || of.row < 0))
                break;
            const RowShare<T> sh(a.logits, of.row, a.V, rank, ranks);
            const int chunks = sh.chunks();
            const int again = kSum && kGrad ? max(0, chunks - kStages) : 0;
            const int end = lane < 8 ? lane : sh.r.tail() + lane - 8;  // warp 0: a value of the ends
            const bool has_end = warp == 0 && lane < 16 &&
                                 (lane < 8 ? rank == 0 && end < sh.r.head : rank == ranks - 1 && end < a.V);
            float M = of.M, Z = of.Z, R = of.R;
            ExpSum rest = of.rest;
            if constexpr (kSum) {
                // ---- the tokens that are not listed
                const uint8_t *const listed = marks + (two ? par * Layout::set : 0);
                const uint32_t *const groups = sm.groups[two ? par : 0];
                Summed sum;
                for (int j = 0; j < chunks; ++j) {
                    const uint32_t k = kb + j, st = k % kStages;
                    wait(&sm.full[st], (k / kStages) & 1);
                    const uint4 *buf = reinterpret_cast<const uint4 *>(smem + st * kChunk);
                    const int n = sh.in_chunk(j);
                    uint4 x[kPer];
                    load_chunk<T>(x, buf, n, no_values<T>());
                    // (most groups of 32 vectors hold no listed token)
                    const uint32_t some[2] = {groups[2 * j] >> warp & 0x10001u,
                                              groups[2 * j + 1] >> warp & 0x10001u};
                    if (!kGrad || j < again) {
                        __syncwarp();
                        if (lane == 0)
                            mbar_arrive(&sm.empty[st]);
                    }
                    if (some[0] | some[1])
#pragma unroll
                        for (int q = 0; q < kPer; ++q)
                            if ((some[q >> 1] >> (16 * (q & 1))) & 1u) {
                                const int at = j * kChunkVecs + tid + q * kMath;
                                leave_out<T>(x[q], E == 8 ? listed[at] : listed[at >> 1] >> (4 * (at & 1)));
                            }
                    sum.add<T, kPer>(x, c);
                }
                sum.settle(c);
                if (has_end && !((of.ends >> lane) & 1u))
                    sum.z.add(to_float(sh.r.row[end]), c);
                __syncwarp();
                rest = warp_sum(sum.z, c);
                if (lane == 0)
                    sm.part[par][warp] = rest;
                named_sync(kBarMath, kMath);
                if (kGrad && tid == 0)
                    mbar_arrive(&sm.swept[par]);
                rest = sm.part[par][lane & 15];
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) {
                    ExpSum p;
                    p.m = __shfl_xor_sync(0xFFFFFFFFu, rest.m, o);
                    p.z = __shfl_xor_sync(0xFFFFFFFFu, rest.z, o);
                    rest.merge(p, c);
                }
                if (ranks > 1) {
                    if (tid == 0)
                        mbar_arrive_expect_tx(&sm.crossed[par], 8 * ranks);
                    if (warp == 0 && lane < ranks)
                        send_sum(&sm.of_rank[par][rank], &sm.crossed[par], lane, rest);
                    wait(&sm.crossed[par], (i >> 1) & 1);
                    rest = sm.of_rank[par][0];
                    for (int q = 1; q < ranks; ++q)
                        rest.merge(sm.of_rank[par][q], c);
                }
                // ---- all tokens, the listed ones among them
                M = fmaxf(rest.m, of.x.m);
                Z = rest.z * ex2_mufu((rest.m - M) * c) + of.x.z * ex2_mufu((of.x.m - M) * c);
                if (!(Z > 0.0f && Z <= FLT_MAX) || !finite_f(M) || of.P != of.P)
                    Z = nan_f();  // (and all that is made of it)
                if (rest.z == 0.0f)
                    R = 0.0f;
                if (rank == 0 && tid == 0) {
                    const float log_z = logf(Z);
                    float loss = of.A;
                    if (of.P != 0.0f)
                        loss += of.P * ((M - of.x.m) * a.inv_t + log_z);
                    if (R > 0.0f)
                        loss += R * (logf(R) - ((rest.m - M) * a.inv_t + logf(rest.z) - log_z));
                    a.loss[of.row] = Z == Z ? loss : Z;
                    if (a.stats_out)
                        a.stats_out[of.row] = make_float4(M, Z, rest.m, rest.z);
                }
                if (!kGrad && tid == 0)  // (what was taught of the row goes too)
                    mbar_arrive(&sm.swept[par]);
            } else if (rest.z == 0.0f) {
                R = 0.0f;
            }
            if constexpr (kGrad) {
                const float scale = of.scale;
                const float r = rest.z * ex2_mufu((rest.m - M) * c) / Z;
                if (tid == 0)
                    sm.fix[par] = make_float4(M, Z, of.P + R, scale);
                // of s_v relative to the reference of the others
                const float f = rest.z == 0.0f ? (Z == Z ? 0.0f : Z) : scale * (r * (of.P + R) - R) / rest.z;
                T *grad = static_cast<T *>(a.grad) + of.row * a.V;
                if (has_end)
                    grad[end] = from_float<T>(ex2_mufu((to_float(sh.r.row[end]) - rest.m) * c) * f);
                uint4 *out = reinterpret_cast<uint4 *>(grad + sh.r.head) + sh.v0;
                const RowTerms terms(rest.m, c, f);
                for (int q = 0; q < chunks; ++q) {
                    // the retained chunks, then those that came again
                    const int j = q < chunks - again ? q + again : q - (chunks - again);
                    const uint32_t k = kb + (q < chunks - again ? j : chunks + j), st = k % kStages;
                    if (!kSum || q >= chunks - again)
                        wait(&sm.full[st], (k / kStages) & 1);
                    const uint4 *buf = reinterpret_cast<const uint4 *>(smem + st * kChunk);
                    const int n = sh.in_chunk(j);
                    uint4 x[kPer];
                    load_chunk<T>(x, buf, n, 0u);
                    __syncwarp();
                    if (lane == 0)
                        mbar_arrive(&sm.empty[st]);
#pragma unroll
                    for (int p = 0; p < kPer; ++p) {
                        const int v = tid + p * kMath;
                        const uint4 y = terms.template of<T>(x[p]);
                        if (v < n)
                            __stcs(out + j * kChunkVecs + v, y);
                    }
                }
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(&sm.written[par]);
            }
            kb += chunks + again;
        }
    } else if (warp < kMathWarps + kTeachers / 32) {
        // ------------------------------------------------------------ the teacher
        constexpr int kMine = kMaxTop / kTeachers;
        const int t = tid - kMath;
        int *const idx = reinterpret_cast<int *>(smem + Layout::dup);
        float *const mass = reinterpret_cast<float *>(idx + kMaxTop);
        RowWalk walk(a.mask, a.rows, true);
        // The lists are read a row ahead: of the row to come, as they lie in memory.
        int64_t next_row;
        int next_v[kMine];
        float next_s[kMine], next_lse = 0.0f, next_scale = 0.0f;
        float4 next_given = make_float4(0, 0, 0, 0);
        auto fetch = [&](uint32_t i) {
            next_row = walk.find(cluster + (int64_t)i * clusters);
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                const int k = t + j * kTeachers;
                next_v[j] = -1;
                next_s[j] = neg_inf_f();
                if (next_row >= 0 && k < a.K) {
                    next_v[j] = a.index[next_row * a.K + k];
                    next_s[j] = top_value(a, next_row * a.K + k);
                }
            }
            if (next_row >= 0) {
                if (a.lse)
                    next_lse = a.lse[next_row];
                if (kGrad)
                    next_scale = a.grad_loss[next_row] * a.inv_t;
                if (!kSum)
                    next_given = a.stats_in[next_row];
            }
        };
        fetch(0);
        int old[kMine];  // of the row before: its listed tokens, and what their gradients need
        float old_p[kMine], old_x[kMine];
        int64_t old_row = -1;
        int older[kMine];  // and of the one before it
        int64_t older_row = -1;
#pragma unroll
        for (int j = 0; j < kMine; ++j)
            old[j] = older[j] = -1, old_p[j] = old_x[j] = 0.0f;
        for (uint32_t i = 0;; ++i) {
            const uint32_t par = i & 1;
            const int64_t row = next_row;
            int v[kMine];
            float m[kMine], x[kMine];
            float P = 0.0f, R = 0.0f, A = 0.0f;
            const float scale = next_scale;
            const float4 given = next_given;
            ExpSum of_x;
            if (row >= 0) {
                const T *logits = static_cast<const T *>(a.logits) + row * a.V;
                const RowShare<T> sh(a.logits, row, a.V, rank, ranks);
                float most = -FLT_MAX;
                T raw[kMine];
#pragma unroll
                for (int j = 0; j < kMine; ++j) {
                    v[j] = next_v[j] >= 0 && next_v[j] < a.V ? next_v[j] : -1;
                    m[j] = v[j] >= 0 ? next_s[j] : neg_inf_f();
                    raw[j] = from_float<T>(0.0f);
                    // In place the gradient takes the logits' place.  Where the row is summed no CTA
                    // writes before all have sent their sums, which come behind these reads; where it
                    // is not, the CTAs of a cluster do not wait for each other, and each reads what it
                    // writes itself, its own share, and no more.
                    if (v[j] >= 0 && (kSum || sh.holds(v[j], rank, ranks)))
                        raw[j] = logits[v[j]];
                }
                const float lse = next_lse;
                fetch(i + 1);
#pragma unroll
                for (int j = 0; j < kMine; ++j)
                    if (j == 0 || j * kTeachers < a.K) {
                        m[j] = score(a, m[j]);
                        most = Most()(most, m[j]);
                    }
                most = a.lse ? lse : teach_reduce(most, sm.reduce[0], Most());
#pragma unroll
                for (int j = 0; j < kMine; ++j)
                    if (j == 0 || j * kTeachers < a.K) {
                        m[j] = v[j] >= 0 ? expf(exponent(a, m[j], most)) : 0.0f;
                        P += m[j];
                    }
                P = teach_reduce(P, sm.reduce[1], Add());
                if (a.lse) {
                    if (kSum)
                        P = most == most ? P : most;  // (a NaN, also where nothing is listed)
                    R = fmaxf(1.0f - P, 0.0f);
                } else if (P != 0.0f) {
#pragma unroll
                    for (int j = 0; j < kMine; ++j)
                        if (j == 0 || j * kTeachers < a.K)
                            m[j] = __fdiv_rn(m[j], P);
                    P = P == P ? 1.0f : P;
                }
#pragma unroll
                for (int j = 0; j < kMine; ++j)
                    x[j] = v[j] >= 0 ? to_float(raw[j]) : neg_inf_f();
            }
            // ---- the marks: those of the row that had this set go, this one's come
            if (kSum && two && i > 1)
                wait(&sm.swept[par], ((i - 2) >> 1) & 1);
            if (kSum && !two && i > 0)
                wait(&sm.swept[par ^ 1], ((i - 1) >> 1) & 1);
            uint8_t *const listed = marks + (two ? par * Layout::set : 0);
            uint32_t *const groups = sm.groups[two ? par : 0];
            if (named_sync_or(kBarTeach, kTeachers, dead))
                break;
            auto mark = [&](const RowShare<T> &sh, int at, bool set) -> bool {  // whether it was set before
                uint32_t *word, bit;
                if (at < sh.r.head) {
                    word = &sm.ends;
                    bit = at;
                } else if (at >= sh.r.tail()) {
                    word = &sm.ends;
                    bit = 8 + at - sh.r.tail();
                } else {
                    const int b = at - sh.r.head - sh.v0 * E;
                    if (b < 0 || b >= (sh.v1 - sh.v0) * E)
                        return false;
                    word = reinterpret_cast<uint32_t *>(listed) + (b >> 5);
                    bit = b & 31;
                    if (set)
                        atomicOr(&groups[b / E >> 10], 1u << (b / E >> 5 & 31));
                }
                if (set)
                    return (atomicOr(word, 1u << bit) >> bit) & 1u;
                atomicAnd(word, ~(1u << bit));
                return false;
            };
            if ((two ? older_row : old_row) >= 0) {
                const RowShare<T> sh(a.logits, two ? older_row : old_row, a.V, rank, ranks);
#pragma unroll
                for (int j = 0; j < kMine; ++j)
                    if ((two ? older[j] : old[j]) >= 0)
                        mark(sh, two ? older[j] : old[j], false);
            }
            if (t == 0) {
                sm.ends = 0;
                sm.twice = 0;
            }
            if (t < kMostListed / 4 / 1024)
                groups[t] = 0;
            named_sync(kBarTeach, kTeachers);
            if (row >= 0) {
                const RowShare<T> sh(a.logits, row, a.V, rank, ranks);
                bool again = false;
#pragma unroll
                for (int j = 0; j < kMine; ++j)
                    if (v[j] >= 0)
                        again |= mark(sh, v[j], true);
                if (ranks > 1) {
                    // the marks are of this CTA's share: other tokens are looked up in a table
                    const int size = a.K <= 64 ? 128 : 2 << (32 - __clz(a.K - 1));
                    for (int q = t; q < size; q += kTeachers)
                        idx[q] = -1;
                    named_sync(kBarTeach, kTeachers);
#pragma unroll
                    for (int j = 0; j < kMine; ++j) {
                        if (v[j] < 0)
                            continue;
                        int h = (int)((uint32_t)v[j] * 2654435761u >> (__clz(size) + 1));
                        for (int q = 0; q < size; ++q, h = (h + 1) & (size - 1)) {
                            const int there = atomicCAS(&idx[h], -1, v[j]);
                            if (there == -1)
                                break;
                            if (there == v[j]) {
                                again = true;
                                break;
                            }
                        }
                    }
                }
                if (again)
                    sm.twice = 1;
                named_sync(kBarTeach, kTeachers);
                if (sm.twice) {
                    // a token listed more than once: its masses count together, in its first place
#pragma unroll
                    for (int j = 0; j < kMine; ++j)
                        if (t + j * kTeachers < a.K) {
                            idx[t + j * kTeachers] = v[j];
                            mass[t + j * kTeachers] = m[j];
                        }
                    named_sync(kBarTeach, kTeachers);
#pragma unroll
                    for (int j = 0; j < kMine; ++j) {
                        const int k = t + j * kTeachers;
                        if (v[j] < 0)
                            continue;
                        m[j] = 0.0f;
                        for (int q = 0; q < a.K; ++q)
                            if (idx[q] == v[j]) {
                                if (q < k) {
                                    v[j] = -1;
                                    break;
                                }
                                m[j] += mass[q];
                            }
                    }
                }
                if constexpr (kSum) {
                    // ---- what is of the listed tokens alone
                    float top = -FLT_MAX;
#pragma unroll
                    for (int j = 0; j < kMine; ++j)
                        if (v[j] >= 0)
                            top = Most()(top, x[j]);
                    top = teach_reduce(top, sm.reduce[0], Most());
                    of_x.m = top;
                    float z = 0.0f;
#pragma unroll
                    for (int j = 0; j < kMine; ++j)
                        if (v[j] >= 0) {
                            z += ex2_mufu((x[j] - top) * c);
                            if (m[j] != 0.0f)
                                A += m[j] * (logf(m[j]) - (x[j] - top) * a.inv_t);
                        }
                    of_x.z = teach_reduce(z, sm.reduce[1], Add());
                    A = teach_reduce(A, sm.reduce[2], Add());
                }
            }
            if (t == 0) {
                Taught &of = sm.taught[par];
                of.row = row;
                of.P = P;
                of.R = R;
                of.A = A;
                of.x = of_x;
                of.scale = scale;
                of.ends = sm.ends;
                of.M = given.x;
                of.Z = given.y;
                of.rest.m = given.z;
                of.rest.z = given.w;
                mbar_arrive(&sm.ready[par]);
            }
            // ---- the gradients of the row before's listed tokens
            if (kGrad && old_row >= 0) {
                wait(&sm.written[par ^ 1], ((i - 1) >> 1) & 1);
                if (!dead) {
                    const float4 fix = sm.fix[par ^ 1];
                    const RowShare<T> sh(a.logits, old_row, a.V, rank, ranks);
                    T *grad = static_cast<T *>(a.grad) + old_row * a.V;
#pragma unroll
                    for (int j = 0; j < kMine; ++j) {
                        const int at = old[j];
                        if (at < 0)
                            continue;
                        if (sh.holds(at, rank, ranks))
                            grad[at] = from_float<T>(
                                fix.w * (ex2_mufu((old_x[j] - fix.x) * c) / fix.y * fix.z - old_p[j]));
                    }
                }
            }
            if (row < 0)
                break;
            older_row = old_row;
            old_row = row;
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                older[j] = old[j];
                old[j] = v[j];
                old_p[j] = m[j];
                old_x[j] = x[j];
            }
        }
    } else if (warp == kMathWarps + kTeachers / 32) {
        // ------------------------------------------------------------ the copies
        const uint64_t policy = make_evict_first_policy();
        RowWalk walk(a.mask, a.rows, true);
        uint32_t k = 0;
        for (uint32_t i = 0; !dead; ++i) {
            const int64_t row = walk.find(cluster + (int64_t)i * clusters);
            if (row < 0)
                break;
            const RowShare<T> sh(a.logits, row, a.V, rank, ranks);
            const int chunks = sh.chunks();
            const int again = kSum && kGrad ? max(0, chunks - kStages) : 0;
            if (lane == 0)
                for (int q = 0; q < chunks + again; ++q, ++k) {
                    const int j = q < chunks ? q : q - chunks;
                    const uint32_t st = k % kStages, n = sh.in_chunk(j) * 16;
                    if (k >= kStages)
                        wait(&sm.empty[st], (k / kStages - 1) & 1);
                    if (dead)
                        break;
                    const void *src = sh.r.vectors() + sh.v0 + j * kChunkVecs;
                    mbar_arrive_expect_tx(&sm.full[st], n);
                    if (q < again)  // (comes again)
                        bulk_copy_g2s(smem + st * kChunk, src, n, &sm.full[st]);
                    else
                        bulk_copy_g2s_hint(smem + st * kChunk, src, n, &sm.full[st], policy);
                }
            dead = __any_sync(0xFFFFFFFFu, dead);
        }
        // nothing may land in this CTA's memory after it has gone
        if (lane == 0)
            for (uint32_t i = k > kStages ? k - kStages : 0; i < k; ++i)
                mbar_wait(&sm.full[i % kStages], (i / kStages) & 1, a.status, kDrainLimitNs);
    } else {
        // ------------------------------------------------------------ positions that do not count
        RowWalk walk(a.mask, a.rows, false);
        for (uint32_t i = 0;; ++i) {
            const int64_t row = walk.find(cluster + (int64_t)i * clusters);
            if (row < 0)
                break;
            if (kSum && rank == 0 && lane == 0) {
                a.loss[row] = 0.0f;
                if (a.stats_out)
                    a.stats_out[row] = make_float4(0, 0, 0, 0);
            }
            if constexpr (kGrad) {
                const RowShare<T> sh(a.grad, row, a.V, rank, ranks);
                T *grad = static_cast<T *>(a.grad) + row * a.V;
                if (rank == 0 && lane < sh.r.head)
                    grad[lane] = from_float<T>(0.0f);
                if (rank == ranks - 1 && sh.r.tail() + lane < a.V)
                    grad[sh.r.tail() + lane] = from_float<T>(0.0f);
                const int64_t bytes = (int64_t)(sh.v1 - sh.v0) * 16;
                uint8_t *p = reinterpret_cast<uint8_t *>(grad + sh.r.head) + (int64_t)sh.v0 * 16;
                for (int64_t o = (int64_t)lane * kZeros; o < bytes; o += 32 * kZeros)
                    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(p + o),
                                 "r"(smem_addr(smem + Layout::zeros)), "r"((uint32_t)min((int64_t)kZeros, bytes - o))
                                 : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
        }
        if constexpr (kGrad)
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (ranks > 1) {  // no CTA leaves while another may send to it
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
}

// CTAs that share a row: one where there are rows for all SMs; more where rows are few, as long as
// shares have a chunk (a step of one row of 126464 tokens in bf16: 11 us, with two chunks 13), or where
// a share's bits would not fit.
int row_ranks(int64_t rows, int V, int es)
{
    int ranks = 1;
    while (ranks < kMaxRanks &&
           (V / ranks > kMostListed - 64 ||
            (rows * ranks * 2 <= sm_count() && (int64_t)V * es / ranks >= 2 * kChunk)))
        ranks *= 2;
    return ranks;
}

template <typename T, bool kSum, bool kGrad>
cudaError_t launch_kind(const DistillArgs &a, cudaStream_t s)
{
    constexpr int es = sizeof(T);
    auto *few = distill_small_kernel<T, kSum, kGrad, 1>;
    auto *many = distill_small_kernel<T, kSum, kGrad, kMaxTop / kThreads>;
    auto *ring = distill_ring_kernel<T, kSum, kGrad>;
    constexpr int kSmem = RingLayout<kSum, kGrad>::bytes;
    static PerDevice ready;
    static std::atomic<int> held[kMaxCacheDevices][4];
    cudaError_t e = ready.once([&] {
        cudaFuncAttributes f;  // (asked for, a kernel is loaded: a capture may be next)
        cudaError_t r = cudaFuncGetAttributes(&f, few);
        if (r == cudaSuccess)
            r = cudaFuncGetAttributes(&f, many);
        if (r == cudaSuccess)
            r = cudaFuncSetAttribute(ring, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        int dev = 0;
        if (r == cudaSuccess && cudaGetDevice(&dev) == cudaSuccess)
            for (int i = 0; i < 4; ++i)
                held[dev][i] = clusters_held(ring, kRingThreads, kSmem, 1 << i);
        return r;
    });
    if (e != cudaSuccess)
        return e;
    if ((int64_t)a.V * es <= (a.rows > sm_count() ? kManyRow : kSmallRow) ||
        (kSum && !kGrad && a.V <= kLossV && a.rows > kFull * sm_count())) {
        // (long rows a CTA each, as SMs have room for them)
        const int64_t most = (int64_t)a.V * es > kSmallRow ? a.rows : (int64_t)sm_count() * 16;
        return launch(a.K <= kThreads ? few : many, dim3((unsigned)(a.rows < most ? a.rows : most)),
                      dim3(kThreads), (size_t)(a.V / 32 + 1) * 4, s, true, a);
    }
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess)
        return e;
    const int ranks = row_ranks(a.rows, a.V, es);
    const int most = held[dev][ranks == 1 ? 0 : ranks == 2 ? 1 : ranks == 4 ? 2 : 3];
    const int clusters = (int)(a.rows < most ? a.rows : most);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(clusters * ranks));
    cfg.blockDim = dim3(kRingThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)ranks, 1, 1};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = plain_launches ? 1 : 2;
    const int two = RingLayout<kSum, kGrad>::wide || a.V / ranks <= kMostListed / 2 - 64;
    return cudaLaunchKernelEx(&cfg, ring, DistillArgs(a), ranks, two);
}

template <typename T>
cudaError_t launch_distill(const DistillArgs &a, bool sum, bool grad, cudaStream_t s)
{
    return sum && grad ? launch_kind<T, true, true>(a, s)
           : sum       ? launch_kind<T, true, false>(a, s)
                       : launch_kind<T, false, true>(a, s);
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

fdllm_status run_distill(DistillArgs &a, int dtype, bool sum, bool grad, void *stream)
{
    a.status = cache_status_word();
    if (!a.status)
        return FDLLM_ERR_CUDA;
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
