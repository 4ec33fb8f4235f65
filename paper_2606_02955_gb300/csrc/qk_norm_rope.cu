// qk_norm_rope.cu -- fdllm_qk_norm_rope: per-head RMS norm of queries and keys and their
// rotary positions over up to four position axes, one pass over the rows.
//
// Bound by memory: each row is read once and written once (4 bytes moved per 16-bit value
// against about 10 operations).  Measured: 16381 tokens of 32 + 8 heads of 128 channels, bf16, three
// axes: 69 us (336 MB, 4.9 TB/s); 32 tokens of 64 heads: 3 us.
#include <cuda_runtime.h>

#include "cache.cuh"

namespace fdllm {
namespace {

constexpr int kMaxPairs = 256;
constexpr int kMaxAxes = 4;
constexpr int kThreads = 256;

struct QkArgs {
    const void *x[2];          // q, k
    const void *weight[2];     // [D] or null
    void *out[2];              // [T, heads, D]
    int64_t token_stride[2];
    int64_t head_stride[2];
    const int32_t *positions;  // [axes, T]
    int T;
    int Hq;
    int H;                     // Hq + Hk
    int D;
    int pairs;
    int interleaved;
    int section_end[kMaxAxes]; // pair p follows the first axis a with p < section_end[a]
    float eps;
    // Turns per position of each pair as a 64-bit fraction of a turn.  position * turn, modulo
    // 2^64, is the angle modulo a full turn exactly: an fp32 product of a position of 10^5 and
    // a frequency is off by 4e-3 radians, a 64-bit fraction by less than 2^-32 turns.
    uint64_t turn[kMaxPairs];
};

// cos and sin of pair p of token t.
__device__ __forceinline__ float2 pair_turn(const QkArgs &a, int t, int p)
{
    int axis = 0;
#pragma unroll
    for (int i = 0; i < kMaxAxes - 1; ++i)
        axis += p >= a.section_end[i] ? 1 : 0;
    const int64_t pos = a.positions[(int64_t)axis * a.T + t];
    const uint64_t phase = (uint64_t)pos * a.turn[p];
    float2 cs;
    sincospif((float)(int32_t)(phase >> 32) * 0x1p-31f, &cs.y, &cs.x);
    return cs;
}

// Rows of D channels, all of them turned, on 16-byte vectors: D / 16 lanes to a row, each
// holding eight pairs, so that a warp has 32 to 64 independent 16-byte loads in flight and the
// norm's sum takes two to four shuffles.  The angles of a CTA's TOKENS tokens are computed
// once into shared memory for all of their heads.
template <typename T, int D, int TOKENS>
__global__ void __launch_bounds__(kThreads) qk_rows_kernel(const __grid_constant__ QkArgs a)
{
    constexpr int kPairs = D / 2;
    constexpr int kLanes = D / 16;
    constexpr int kGroups = kThreads / kLanes;
    __shared__ __align__(16) float2 cs[TOKENS * kPairs];
    pdl_wait();
    const int64_t t0 = (int64_t)blockIdx.x * TOKENS;
    const int tokens = (int)min((int64_t)TOKENS, a.T - t0);
    for (int i = threadIdx.x; i < tokens * kPairs; i += kThreads)
        cs[i] = pair_turn(a, (int)t0 + i / kPairs, i % kPairs);
    __syncthreads();

    const int r = threadIdx.x % kLanes;
    const int e0 = a.interleaved ? 16 * r : 8 * r;
    const int e1 = a.interleaved ? 16 * r + 8 : 8 * r + kPairs;
    const int rows = tokens * a.H;
    // Every lane of a warp runs the same number of turns (the shuffles below need them all).
    for (int base = 0; base < rows; base += kGroups) {
        const int row = base + threadIdx.x / kLanes;
        const bool live = row < rows;
        const int tok = live ? row / a.H : 0;
        const int head = live ? row - tok * a.H : 0;
        const int w = head < a.Hq ? 0 : 1;
        const int h = w ? head - a.Hq : head;
        const T *x = static_cast<const T *>(a.x[w]) + (t0 + tok) * a.token_stride[w] +
                     h * a.head_stride[w];
        float u[8] = {}, v[8] = {};
        if (live) {
            load8(x + e0, u);
            load8(x + e1, v);
        }
        const T *weight = static_cast<const T *>(a.weight[w]);
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            ss += u[i] * u[i] + v[i] * v[i];
#pragma unroll
        for (int m = kLanes / 2; m > 0; m >>= 1)
            ss += __shfl_xor_sync(0xFFFFFFFFu, ss, m);
        if (!live)
            continue;
        if (weight) {
            const float inv = rsqrtf(ss * (1.0f / D) + a.eps);
            float wu[8], wv[8];
            load8(weight + e0, wu);
            load8(weight + e1, wv);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[i] *= inv * wu[i];
                v[i] *= inv * wv[i];
            }
        }
        const float4 *c4 = reinterpret_cast<const float4 *>(cs + tok * kPairs + 8 * r);
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 f = c4[i];
            c[2 * i] = f.x, s[2 * i] = f.y, c[2 * i + 1] = f.z, s[2 * i + 1] = f.w;
        }
        float y[8], z[8];
        if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[2 * i] = u[2 * i] * c[i] - u[2 * i + 1] * s[i];
                y[2 * i + 1] = u[2 * i + 1] * c[i] + u[2 * i] * s[i];
                z[2 * i] = v[2 * i] * c[i + 4] - v[2 * i + 1] * s[i + 4];
                z[2 * i + 1] = v[2 * i + 1] * c[i + 4] + v[2 * i] * s[i + 4];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = u[i] * c[i] - v[i] * s[i];
                z[i] = v[i] * c[i] + u[i] * s[i];
            }
        }
        T *o = static_cast<T *>(a.out[w]) + ((t0 + tok) * (w ? a.H - a.Hq : a.Hq) + h) * D;
        store8(o + e0, y);
        store8(o + e1, z);
    }
}

// Any even D, any number of pairs, any alignment: one warp to a row, one token to a CTA.  A row
// is read twice (the second time from L1).
template <typename T>
__global__ void __launch_bounds__(kThreads) qk_any_kernel(const __grid_constant__ QkArgs a)
{
    __shared__ float2 cs[kMaxPairs];
    pdl_wait();
    const int64_t t = blockIdx.x;
    for (int p = threadIdx.x; p < a.pairs; p += kThreads)
        cs[p] = pair_turn(a, (int)t, p);
    __syncthreads();
    const int lane = threadIdx.x & 31;
    for (int head = threadIdx.x >> 5; head < a.H; head += kThreads / 32) {
        const int w = head < a.Hq ? 0 : 1;
        const int h = w ? head - a.Hq : head;
        const T *x = static_cast<const T *>(a.x[w]) + t * a.token_stride[w] +
                     h * a.head_stride[w];
        const T *weight = static_cast<const T *>(a.weight[w]);
        T *o = static_cast<T *>(a.out[w]) + (t * (w ? a.H - a.Hq : a.Hq) + h) * a.D;
        float inv = 1.0f;
        if (weight) {
            float ss = 0.0f;
            for (int i = lane; i < a.D; i += 32) {
                const float f = to_float(x[i]);
                ss += f * f;
            }
#pragma unroll
            for (int m = 16; m > 0; m >>= 1)
                ss += __shfl_xor_sync(0xFFFFFFFFu, ss, m);
            inv = rsqrtf(ss / a.D + a.eps);
        }
        for (int p = lane; p < a.pairs; p += 32) {
            const int i = a.interleaved ? 2 * p : p;
            const int j = a.interleaved ? 2 * p + 1 : p + a.pairs;
            float u = to_float(x[i]), v = to_float(x[j]);
            if (weight) {
                u *= inv * to_float(weight[i]);
                v *= inv * to_float(weight[j]);
            }
            o[i] = from_float<T>(u * cs[p].x - v * cs[p].y);
            o[j] = from_float<T>(v * cs[p].x + u * cs[p].y);
        }
        for (int i = 2 * a.pairs + lane; i < a.D; i += 32) {
            float u = to_float(x[i]);
            if (weight)
                u *= inv * to_float(weight[i]);
            o[i] = from_float<T>(u);
        }
    }
}

// Four tokens to a CTA share one pass of angles where that leaves a few CTAs for every SM;
// fewer tokens take one CTA each, so that a short block still spreads over the SMs (40 heads: 32
// tokens 3.1 us, in fours 5.7; 2048 tokens 11.7 both ways; 8192 tokens in fours 37.4, one by one 45.9).
constexpr int kManyTokens = 4 * 1024;

template <typename T, int D>
cudaError_t launch_rows(const QkArgs &a, cudaStream_t s)
{
    if (a.T >= kManyTokens)
        return launch(qk_rows_kernel<T, D, 4>, dim3((a.T + 3) / 4), dim3(kThreads), 0, s, true, a);
    return launch(qk_rows_kernel<T, D, 1>, dim3(a.T), dim3(kThreads), 0, s, true, a);
}

template <typename T>
cudaError_t launch_qk(const QkArgs &a, bool vectors, cudaStream_t s)
{
    if (vectors && 2 * a.pairs == a.D) {
        if (a.D == 64)
            return launch_rows<T, 64>(a, s);
        if (a.D == 128)
            return launch_rows<T, 128>(a, s);
        if (a.D == 256)
            return launch_rows<T, 256>(a, s);
    }
    return launch(qk_any_kernel<T>, dim3(a.T), dim3(kThreads), 0, s, true, a);
}

}  // namespace
}  // namespace fdllm

using namespace fdllm;

extern "C" fdllm_status fdllm_qk_norm_rope(
    const void *q, const int64_t *q_strides, const void *k, const int64_t *k_strides, int dtype,
    int T, int Hq, int Hk, int D, const void *q_weight, const void *k_weight, double eps,
    const int32_t *positions, int axes, const int32_t *sections, const double *inv_freq,
    int pairs, int interleaved, void *out_q, void *out_k, void *stream)
{
    if (dtype != FDLLM_BF16 && dtype != FDLLM_FP16 && dtype != FDLLM_FP32)
        return FDLLM_ERR_ARG;
    if (T < 0 || Hq < 1 || Hk < 0 || (int64_t)Hq + Hk > 65536 || D < 2 || D > 2 * kMaxPairs ||
        D % 2 != 0 || pairs < 0 || 2 * pairs > D || axes < 1 || axes > kMaxAxes ||
        (interleaved != 0 && interleaved != 1) || !std::isfinite(eps) || eps < 0.0)
        return FDLLM_ERR_ARG;
    if (!q_strides || (Hk > 0 && !k_strides) || (pairs > 0 && !inv_freq) ||
        (axes > 1 && !sections))
        return FDLLM_ERR_ARG;
    QkArgs a;
    int end = 0;
    for (int i = 0; i < kMaxAxes; ++i) {
        if (i < axes) {
            const int n = sections ? sections[i] : pairs;
            if (n < 0 || n > pairs)
                return FDLLM_ERR_ARG;
            end += n;
        }
        a.section_end[i] = i < axes - 1 ? end : kMaxPairs;
    }
    if (end != pairs)
        return FDLLM_ERR_ARG;
    for (int p = 0; p < pairs; ++p) {
        if (!std::isfinite(inv_freq[p]))
            return FDLLM_ERR_ARG;
        // radians -> turns, modulo 1, as a 64-bit fraction (a double holds 53 bits of it)
        double turns = inv_freq[p] / 6.283185307179586476925286766559;
        turns -= std::floor(turns);
        const double scaled = std::ldexp(turns, 64);
        a.turn[p] = scaled >= 18446744073709551616.0 ? 0u : (uint64_t)scaled;
    }
    if (T == 0)
        return FDLLM_OK;
    if (!q || !out_q || (Hk > 0 && (!k || !out_k)) || !positions)
        return FDLLM_ERR_ARG;
    const int es = dtype == FDLLM_FP32 ? 4 : 2;
    const int64_t zero[2] = {0, 0};
    bool vectors = aligned16(q, q_strides, 2, es) && aligned16(out_q, zero, 0, es) &&
                   aligned16(q_weight, zero, 0, es) && aligned16(k_weight, zero, 0, es);
    if (Hk > 0)
        vectors = vectors && aligned16(k, k_strides, 2, es) && aligned16(out_k, zero, 0, es);
    a.x[0] = q;
    a.x[1] = k;
    a.weight[0] = q_weight;
    a.weight[1] = k_weight;
    a.out[0] = out_q;
    a.out[1] = out_k;
    a.token_stride[0] = q_strides[0];
    a.head_stride[0] = q_strides[1];
    a.token_stride[1] = Hk > 0 ? k_strides[0] : 0;
    a.head_stride[1] = Hk > 0 ? k_strides[1] : 0;
    a.positions = positions;
    a.T = T;
    a.Hq = Hq;
    a.H = Hq + Hk;
    a.D = D;
    a.pairs = pairs;
    a.interleaved = interleaved;
    a.eps = (float)eps;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == FDLLM_BF16)
        e = launch_qk<__nv_bfloat16>(a, vectors, s);
    else if (dtype == FDLLM_FP16)
        e = launch_qk<__half>(a, vectors, s);
    else
        e = launch_qk<float>(a, vectors, s);
    return e == cudaSuccess ? FDLLM_OK : FDLLM_ERR_CUDA;
}
