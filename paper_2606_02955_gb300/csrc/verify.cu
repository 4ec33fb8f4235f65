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
#include <cuda_runtime.h>

#include "vocab_rows.cuh"

namespace fdllm {
namespace {

constexpr int kMaxNodes = FDLLM_MAX_L;
constexpr int kThreads = 512;

struct VerifyArgs {
    const void *target;       // [B, M, V]
    const void *draft;        // [B, M - 1, V] or null
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
    UnitPartial *partials;    // [B, M] of the target's rows, [B, M - 1] of the draft's
};

__device__ __forceinline__ int nodes_of(const VerifyArgs &a, int b)
{
    return a.lens ? min(max(a.lens[b], 1), a.M) : a.M;
}

// One CTA a row: maximum, its first index, and the sum relative to it.
template <typename T>
__global__ void __launch_bounds__(kThreads) verify_rows_kernel(const __grid_constant__ VerifyArgs a)
{
    constexpr int E = 16 / sizeof(T);
    __shared__ ExpSum sums[kThreads / 32];
    __shared__ uint32_t firsts[kThreads / 32];
    pdl_wait();
    const int64_t targets = (int64_t)a.B * a.M, rows = targets + (a.draft ? (int64_t)a.B * (a.M - 1) : 0);
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const bool of_draft = row >= targets;
        const int64_t at = of_draft ? row - targets : row;
        const int per = of_draft ? a.M - 1 : a.M;
        const int b = (int)(at / per), j = (int)(at - (int64_t)b * per);
        if (j >= nodes_of(a, b) - (of_draft ? 1 : 0))
            continue;
        const float c = of_draft ? a.cd : a.ct;
        const RowSpan<T> s(static_cast<const T *>(of_draft ? a.draft : a.target) + at * a.V, a.V);
        ExpSum z;
        uint32_t first = kNoIdx;
        auto one = [&](int i) {
            const float x = to_float(s.row[i]);
            if (x > z.m || (x == z.m && (uint32_t)i < first))
                first = i;
            z.add(x, c);
        };
        for (int i = threadIdx.x; i < s.vecs; i += kThreads) {
            float y[E];
            widen<T>(s.vectors()[i], y);
            float top = y[0];
#pragma unroll
            for (int e = 1; e < E; ++e)
                top = fmaxf(top, y[e]);
            if (top > z.m || first == kNoIdx) {
#pragma unroll
                for (int e = E - 1; e >= 0; --e)
                    if (y[e] == top && top >= z.m)
                        first = s.head + i * E + e;
                z.raise(top, c);
            }
#pragma unroll
            for (int e = 0; e < E; ++e)
                z.z += ex2_mufu((y[e] - z.m) * c);
        }
        for (int i = threadIdx.x; i < s.head; i += kThreads)
            one(i);
        for (int i = s.tail() + threadIdx.x; i < a.V; i += kThreads)
            one(i);
        const float top = warp_most(z.m);
        first = __reduce_min_sync(0xFFFFFFFFu, z.m == top ? first : kNoIdx);
        z = warp_sum(z, c);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) {
            sums[threadIdx.x >> 5] = z;
            firsts[threadIdx.x >> 5] = first;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kThreads / 32; ++w) {
                if (sums[w].m > z.m || (sums[w].m == z.m && firsts[w] < first))
                    first = firsts[w];
                z.merge(sums[w], c);
            }
            UnitPartial p;
            p.M = z.m;
            p.S = z.z;
            p.idx = first;
            p.pad = 0;
            a.partials[row] = p;
        }
    }
}

// One CTA a sequence: the walk, then the draw.
template <typename T>
__global__ void __launch_bounds__(kThreads) verify_walk_kernel(const __grid_constant__ VerifyArgs a)
{
    __shared__ float take[kMaxNodes];   // p of a node's token after its parent
    __shared__ float drawn[kMaxNodes];  // q of it
    __shared__ short parent[kMaxNodes];
    __shared__ uint8_t bad[kMaxNodes];
    __shared__ int path[kMaxNodes + 1];
    __shared__ int cur, taken, failed, rejected;
    __shared__ unsigned long long best[kThreads / 32];
    extern __shared__ __align__(16) uint32_t gone[];  // tokens of the last node's children
    pdl_wait();
    const int b = blockIdx.x, tid = threadIdx.x, n = nodes_of(a, b);
    const int64_t base = (int64_t)b * a.M, dbase = (int64_t)a.B * a.M + (int64_t)b * (a.M - 1);
    const T *target = static_cast<const T *>(a.target) + base * a.V;
    const T *draft = static_cast<const T *>(a.draft) + (int64_t)b * (a.M - 1) * a.V;
    const UnitPartial *tp = a.partials + base, *dp = a.partials + dbase;
    auto fine = [](const UnitPartial &p) {
        return p.S > 0.0f && p.S <= FLT_MAX && finite_f(p.M);
    };
    if (!a.greedy)
        for (int i = tid; i < (a.V + 31) / 32; i += kThreads)
            gone[i] = 0;
    for (int j = tid; j < n; j += kThreads) {
        bad[j] = !fine(tp[j]) || (a.draft && j < n - 1 && !fine(dp[j]));
        const int pa = j == 0 ? -1 : a.parents ? a.parents[base + j] : j - 1;
        const bool hung = pa >= 0 && pa < j;
        parent[j] = hung ? pa : -1;
        take[j] = drawn[j] = 0.0f;
        const int d = a.tokens[base + j];
        if (!hung || d < 0 || d >= a.V)
            continue;
        if (a.greedy) {
            take[j] = tp[pa].idx == (uint32_t)d ? 1.0f : 0.0f;
            continue;
        }
        const float x = to_float(target[(int64_t)pa * a.V + d]);
        take[j] = ex2_mufu((x - tp[pa].M) * a.ct) / tp[pa].S;
        if (a.draft) {
            const float y = to_float(draft[(int64_t)pa * a.V + d]);
            drawn[j] = ex2_mufu((y - dp[pa].M) * a.cd) / dp[pa].S;
        } else {
            for (int i = 1; i < j; ++i)
                if (a.tokens[base + i] == d && (a.parents ? a.parents[base + i] : i - 1) == pa)
                    take[j] = 0.0f;  // its token is gone with the sibling before it
        }
    }
    __syncthreads();
    if (tid == 0) {
        int at = 0, len = 0, wrong = bad[0], stop = 0;
        double left = 1.0;
        path[0] = 0;
        for (int j = 1; j < n && !wrong && !stop; ++j) {
            if (parent[j] != at)
                continue;
            bool ok;
            if (a.greedy)
                ok = take[j] != 0.0f;
            else if (a.draft)
                ok = (double)a.uniform[base + j] * drawn[j] < take[j];
            else
                ok = (double)a.uniform[base + j] * left < take[j];
            if (ok) {
                at = j;
                path[++len] = j;
                left = 1.0;
                wrong = bad[j];
            } else {
                left -= take[j];
                stop = a.draft != nullptr;
            }
        }
        cur = at;
        taken = len;
        failed = wrong;
        rejected = stop;
    }
    __syncthreads();
    int extra = -1;
    if (!failed) {
        const UnitPartial p = tp[cur];
        extra = (int)p.idx;
        if (!a.greedy) {
            if (!a.draft)
                for (int j = 1 + tid; j < n; j += kThreads) {
                    const int d = a.tokens[base + j];
                    if (parent[j] == cur && d >= 0 && d < a.V)
                        atomicOr(&gone[d >> 5], 1u << (d & 31));
                }
            __syncthreads();
            const T *row = target + (int64_t)cur * a.V, *drow = draft + (int64_t)cur * a.V;
            const float *noise = a.noise + (int64_t)b * a.V;
            UnitPartial q = {};
            if (rejected)
                q = dp[cur];
            unsigned long long top = 0;
            for (int turn = 0; turn < 2 && top == 0; ++turn) {  // the second: from p itself
                for (int v = tid; v < a.V; v += kThreads) {
                    float r = ex2_mufu((to_float(row[v]) - p.M) * a.ct) / p.S;
                    if (turn == 0 && rejected)
                        r = fmaxf(r - ex2_mufu((to_float(drow[v]) - q.M) * a.cd) / q.S, 0.0f);
                    if (turn == 0 && (gone[v >> 5] >> (v & 31)) & 1u)
                        r = 0.0f;
                    const float key = __fdiv_rn(r, noise[v]);
                    if (r > 0.0f && key > 0.0f) {
                        const unsigned long long k =
                            ((unsigned long long)__float_as_uint(key) << 32) | (0xFFFFFFFFu - v);
                        top = k > top ? k : top;
                    }
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    const unsigned long long k = __shfl_xor_sync(0xFFFFFFFFu, top, o);
                    top = k > top ? k : top;
                }
                __syncthreads();
                if ((tid & 31) == 0)
                    best[tid >> 5] = top;
                __syncthreads();
                for (int w = 0; w < kThreads / 32; ++w)
                    top = best[w] > top ? best[w] : top;
            }
            if (top)
                extra = (int)(0xFFFFFFFFu - (uint32_t)top);
        }
    }
    for (int j = tid; j < a.M; j += kThreads) {
        int token = -1, node = -1;
        if (!failed && j <= taken) {
            node = path[j];
            token = j < taken ? a.tokens[base + path[j + 1]] : extra;
        }
        a.out_tokens[base + j] = token;
        a.out_nodes[base + j] = node;
    }
    if (tid == 0)
        a.out_n[b] = failed ? FDLLM_ROW_NONFINITE : taken;
}

template <typename T>
cudaError_t launch_verify(const VerifyArgs &a, cudaStream_t s)
{
    static PerDevice ready;
    cudaError_t e = ready.once([] {
        return cudaFuncSetAttribute(verify_walk_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    kMaxRowV / 8);
    });
    if (e != cudaSuccess)
        return e;
    const int64_t rows = (int64_t)a.B * (a.draft ? 2 * a.M - 1 : a.M), most = (int64_t)sm_count() * 4;
    e = launch(verify_rows_kernel<T>, dim3((unsigned)(rows < most ? rows : most)), dim3(kThreads), 0, s,
               true, a);
    if (e != cudaSuccess)
        return e;
    return launch(verify_walk_kernel<T>, dim3(a.B), dim3(kThreads),
                  a.greedy ? 0 : (size_t)((a.V + 31) / 32) * 4, s, true, a);
}

size_t verify_bytes(int B, int M)
{
    return ((size_t)B * (2 * (size_t)M - 1) * sizeof(UnitPartial) + 255) / 256 * 256;
}

bool verify_sizes(int B, int M, int V)
{
    return B >= 1 && B <= kMaxGridYZ && M >= 1 && M <= kMaxNodes && V >= 1 && V <= kMaxRowV;
}

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" {

size_t fdllm_verify_draft_workspace_bytes(int B, int M, int V, int dtype)
{
    return verify_sizes(B, M, V) && rows_dtype(dtype) ? verify_bytes(B, M) : 0;
}

fdllm_status fdllm_verify_draft(const void *target, const void *draft, int dtype, int B, int M,
                                int V, const int32_t *tokens, const int32_t *parents,
                                const int32_t *lens, double temperature, double draft_temperature,
                                const float *uniform, const float *noise, int32_t *out_tokens,
                                int32_t *out_nodes, int32_t *out_n, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    const bool greedy = temperature == 0.0;
    auto sane = [](double t) { return t >= 1e-6 && t <= 1e6; };
    if (!verify_sizes(B, M, V) || !rows_dtype(dtype) || !target || !tokens || !out_tokens ||
        !out_nodes || !out_n || (!greedy && (!sane(temperature) || !uniform || !noise)) ||
        (draft && (greedy || parents || !sane(draft_temperature))))
        return FDLLM_ERR_ARG;
    if (((reinterpret_cast<uintptr_t>(target) | reinterpret_cast<uintptr_t>(draft) |
          reinterpret_cast<uintptr_t>(noise)) & 15u) != 0)
        return FDLLM_ERR_ALIGN;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
        workspace_bytes < verify_bytes(B, M))
        return FDLLM_ERR_WORKSPACE;
    VerifyArgs a = {};
    a.target = target;
    a.draft = M > 1 ? draft : nullptr;
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
    a.partials = static_cast<UnitPartial *>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == FDLLM_BF16   ? launch_verify<__nv_bfloat16>(a, s)
                          : dtype == FDLLM_FP16 ? launch_verify<__half>(a, s)
                                                : launch_verify<float>(a, s);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}

}  // extern "C"
