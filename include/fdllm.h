/*
 * fdllm.h -- C interface of the GB300 (sm_103a) commit-set selection library for
 * Frechet profile decoding of masked diffusion LLMs (Fast-dLLM++).
 *
 * One decode step of the paper's Algorithm 1, from logits at the masked positions of the
 * active block to the committed tokens and the updated mask:
 *   (a1) per masked position i: x_hat_i = argmax_v p_i(v) (lowest v on ties) and the
 *        confidence c_i = max_v p_i(v) = exp(M_i - logsumexp_i), p_i = softmax of row i
 *        (Sec. 3 "Notation"; Alg. 1 confidence loop);
 *   (a2) sort the masked confidences of each batch row in descending order, equal
 *        confidences lower position first (Alg. 1 sort);
 *   (a3) for every prefix size n: L_n = max{0, sum_{j<=n} c_(j) - (n-1)}, U_n = 1 - c_(n),
 *        G_n = L_n - U_n (Sec. 3 "Frechet profile quantities", Eq. frechet_Ln_Un);
 *   (a4) n* = max{n : G_n > delta}, n* = 1 when no n qualifies (Sec. 3; Alg. 1 select);
 *   (a5) reveal the n* most confident masked positions (Alg. 1 reveal).
 * Fast-dLLM's rules are available as alternative modes: factor, accept n iff
 * (n+1)(1 - c_(n)) < f (Sec. 1, Cor. factor-reduction); threshold, commit {i : c_i >= tau}
 * or the single most confident position when that set is empty (Sec. 2).
 *
 * Conventions for every entry point:
 *   - Pointers named logits, mask, out_*, conf, argmax and workspace are DEVICE pointers
 *     owned by the caller; the library never frees them.  `stream` is a cudaStream_t
 *     (NULL = legacy default stream) passed as void* so this header needs no CUDA headers.
 *   - logits is [B, L, V] row-major with V contiguous; dtype FDLLM_BF16 (bfloat16),
 *     FDLLM_FP16 (IEEE half) or FDLLM_FP32.  The base must be 16-byte aligned and
 *     V * sizeof(dtype) a multiple of 16 (V % 8 == 0 for bf16 and fp16, V % 4 == 0 for
 *     fp32); otherwise FDLLM_ERR_ALIGN.  A vocabulary
 *     that is not a multiple can be padded with -inf columns, which change nothing.
 *   - mask is uint8 [B, L], nonzero = masked.  Only masked positions are read from logits.
 *   - Limits: 1 <= B, 1 <= L <= FDLLM_MAX_L, B * L <= FDLLM_MAX_ROWS, V >= 1.
 *   - Work is enqueued asynchronously on `stream`; the return value reports only argument
 *     and launch errors, detected on the host.  Per-row data errors are reported in out_n
 *     (see FDLLM_ROW_NONFINITE) and, for calls that use a workspace, in its sticky status
 *     word, which fdllm_device_status / fdllm_workspace_status / fdllm_static_status read
 *     as FDLLM_ERR_NONFINITE.
 *   - All kernels are deterministic: the same inputs on the same GPU model give
 *     bit-identical outputs.  A position's confidence depends only on its logits and the
 *     call's shape (B * L, V, dtype), which fix how rows are cut into reduction units, so
 *     identical rows of one call give identical confidences (exact ties stay ties).
 *   - Arithmetic: confidences are reduced in fp32 (relative error within 1e-5 of the exact
 *     value); the rules are evaluated on those fp32 confidences with exact 64-bit fixed-point
 *     prefix sums of 1 - c in units of 2^-52 (delta = 1 - f formed from the same integer as
 *     f, so a flat profile gives the factor rule's decision bit for bit), and the threshold
 *     compares c with the smallest fp32 value >= tau, which decides c >= tau exactly.
 */
#ifndef FDLLM_H
#define FDLLM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FDLLM_MAX_L 1024       /* positions per batch row (one CTA sorts a row in smem) */
#define FDLLM_MAX_ROWS 65536   /* B * L: masked-row compaction lives in shared memory */

typedef enum { FDLLM_BF16 = 0, FDLLM_FP32 = 1, FDLLM_FP16 = 2 } fdllm_dtype;

typedef enum {
    FDLLM_PROFILE = 0,   /* Frechet profile rule, Sec. 3: param = f, margin delta = 1 - f */
    FDLLM_FACTOR = 1,    /* Fast-dLLM factor rule: param = f                              */
    FDLLM_THRESHOLD = 2  /* Fast-dLLM threshold rule: param = tau                         */
} fdllm_mode;

typedef enum {
    FDLLM_OK = 0,
    FDLLM_ERR_ARG = 1,       /* a null pointer, a size out of range, an unknown enum, a
                                non-finite param                                         */
    FDLLM_ERR_ALIGN = 2,     /* logits base not 16-byte aligned or V*sizeof(dtype) % 16 */
    FDLLM_ERR_NONFINITE = 3, /* a selection met a row of FDLLM_ROW_NONFINITE (status word) */
    FDLLM_ERR_CUDA = 4,      /* a CUDA runtime call or kernel launch failed             */
    FDLLM_ERR_WORKSPACE = 5, /* caller workspace too small or misaligned                */
    FDLLM_ERR_DEVICE = 6     /* a kernel's bounded wait gave up (see fdllm_device_status) */
} fdllm_status;

/* out_n value of a batch row whose masked logits are unusable: a NaN anywhere in a masked
 * position's row, or a maximum of +inf or -inf.  Such a row commits nothing and its mask
 * is left unchanged; a call with a workspace also records it in the workspace's status word
 * (FDLLM_ERR_NONFINITE from the status calls).  (The paper defines confidences only for
 * proper distributions.) */
#define FDLLM_ROW_NONFINITE (-1)
/* out_n value of every row when a kernel of the step gave up a bounded wait. */
#define FDLLM_ROW_DEVICE_ERROR (-2)

/* ---------------------------------------------------------------------------------- */
/* One whole selection step (steps a1-a5 above; Alg. 1 from the model's logits to the
 * reveal), with a workspace the library owns.
 *
 *   logits      [B, L, V] device, dtype as given, read only at masked positions.
 *   mask        [B, L] uint8 device, nonzero = masked.  UPDATED IN PLACE: committed
 *               positions become 0 (Alg. 1 reveal).
 *   param       profile: f, the rule accepts n iff G_n > delta with delta = 1 - f (the
 *               matched parameter of Cor. factor-reduction; the paper's operating point
 *               delta = 0.25 is f = 0.75).  factor: f.  threshold: tau.  Any finite value
 *               is accepted; the paper states delta in [0, 1] (f in [0, 1]).
 *   out_tokens  [B, L] int32 device: written ONLY at committed positions, with x_hat.
 *   out_commit  [B, L] uint8 device: fully written, 1 = committed this step.
 *   out_n       [B] int32 device: number committed in each row; 0 iff the row had no
 *               masked position; FDLLM_ROW_NONFINITE / FDLLM_ROW_DEVICE_ERROR as above.
 *
 * The library's workspace is allocated on the current device at the first call that
 * needs more than it holds (cudaMalloc, which synchronises), then reused; make one call
 * of the largest shape before capturing the step in a CUDA graph.  Calls that share the
 * library workspace must be ordered on the GPU (one stream, or events); for concurrent
 * steps use fdllm_select_ws with a workspace per stream. */
fdllm_status fdllm_select(const void *logits, int dtype, int B, int L, int V, uint8_t *mask,
                          double param, int mode, int32_t *out_tokens, uint8_t *out_commit,
                          int32_t *out_n, void *stream);

/* Bytes of caller workspace fdllm_select_ws needs for this shape (a pure host function). */
size_t fdllm_workspace_bytes(int B, int L, int V, int dtype);

/* fdllm_select with a caller-provided workspace (device, 256-byte aligned, at least
 * fdllm_workspace_bytes(B, L, V, dtype) bytes).  The workspace must be zero-filled before
 * its first use; every call that completes leaves it ready for the next call, so it is
 * zeroed once, not per call.  The library never allocates on this path. */
fdllm_status fdllm_select_ws(const void *logits, int dtype, int B, int L, int V, uint8_t *mask,
                             double param, int mode, int32_t *out_tokens, uint8_t *out_commit,
                             int32_t *out_n, void *workspace, size_t workspace_bytes,
                             void *stream);

/* The profile rule on calibration-robust confidences (App. C, "Calibration-Robust Frechet
 * Certificates"): every masked confidence c_hat is replaced by the lower confidence
 * c_low = max{0, c_hat - eta_i} (Eq. robust_L_U), the masked positions are ranked by c_low
 * (ties: lower position first), L_eta(n) = max{0, sum_{j<=n} c_low_(j) - (n-1)},
 * U_eta(n) = 1 - c_low_(n), n is accepted iff L_eta(n) - U_eta(n) > delta = 1 - param, and
 * n* = max accepted, or 1 (the paper defines the robust certificate; this selection rule on
 * it is the library's reading).  With uniform eta and no clipping the score is the plain
 * one minus (n+1) eta (Cor. calibration-penalty).
 *   eta               uniform allowance, finite and >= 0 (App. C; otherwise FDLLM_ERR_ARG),
 *                     used when eta_per_position is NULL.
 *   eta_per_position  [B, L] fp32 device array of per-position allowances, or NULL; a
 *                     negative or NaN entry is read as 0 (device data: not checked on the
 *                     host).
 * Everything else as fdllm_select (the same library workspace).  eta = 0 gives exactly
 * fdllm_select's profile rule. */
fdllm_status fdllm_select_robust(const void *logits, int dtype, int B, int L, int V,
                                 uint8_t *mask, double param, double eta,
                                 const float *eta_per_position, int32_t *out_tokens,
                                 uint8_t *out_commit, int32_t *out_n, void *stream);

/* Scratch of fdllm_select_static: a fixed device array of this many bytes. */
#define FDLLM_STATIC_SCRATCH_BYTES (8u << 20)

/* fdllm_select without any allocation, for callers that must not allocate device memory
 * while they run steps: a serving process that reserves all of its memory up front and
 * forbids allocation afterwards, code running under an external allocator that owns the
 * device (a framework's memory pool, a fixed memory budget), or a caller that cannot hand
 * the library a workspace of its own.  (The paper has no counterpart: this is a property
 * of the library, not of the method.)
 *
 * Arguments and results are exactly those of fdllm_select.  The scratch memory is a fixed
 * array of FDLLM_STATIC_SCRATCH_BYTES bytes compiled into the library; every GPU that loads
 * the library holds it until the process exits.  A shape whose scratch need,
 * fdllm_workspace_bytes(B, L, V, dtype), exceeds that size is rejected with
 * FDLLM_ERR_WORKSPACE before anything is enqueued.  8 MiB covers, for example, every shape
 * with V <= 126464 in any dtype (up to B * L = 65536 rows), and fp32 V = 2^20 up to
 * B * L = 16383 rows.
 * The call allocates nothing: no cudaMalloc, no cudaFree, no allocating library routine.
 *
 * The first call on a device looks up the array's device address (cudaGetSymbolAddress)
 * with that device current and caches it; make that first call before any stream capture.
 * Every call clears the array's status word and work counter on `stream` before its
 * kernels run.  All calls on a device share the one array, which keeps the last call's
 * contents: calls whose work overlaps on the GPU (different streams without ordering
 * between them) race on it and produce wrong results; order such calls on one stream or
 * with events. */
fdllm_status fdllm_select_static(const void *logits, int dtype, int B, int L, int V,
                                 uint8_t *mask, double param, int mode, int32_t *out_tokens,
                                 uint8_t *out_commit, int32_t *out_n, void *stream);

/* The sticky device error of fdllm_select_static's array on the current device, as
 * fdllm_device_status reports the library workspace's: synchronises `stream`, returns
 * FDLLM_ERR_DEVICE if a kernel of a static call gave up a bounded wait (every row of that
 * call also reports out_n = -2), else FDLLM_ERR_NONFINITE if its selection found a row of
 * FDLLM_ROW_NONFINITE, FDLLM_OK otherwise, and clears the status.  Call it after a
 * static call and before the next one, which clears the array's status word itself.
 * Allocates nothing. */
fdllm_status fdllm_static_status(void *stream);

/* Step a1 alone (Sec. 3 "Notation"; Alg. 1 confidence loop): for every masked position,
 * out_conf = c = max softmax probability (fp32) and out_argmax = x_hat (int32, lowest index
 * among equal maxima).  Both [B, L] device arrays, written only at masked positions; a
 * row with non-finite logits (see FDLLM_ROW_NONFINITE) gets out_conf = NaN and
 * out_argmax = -1.  Uses the library workspace like fdllm_select. */
fdllm_status fdllm_confidence(const void *logits, int dtype, int B, int L, int V,
                              const uint8_t *mask, float *out_conf, int32_t *out_argmax,
                              void *stream);

/* Step a1's vocabulary reduction alone: the per-unit (max, sum of exp, first index)
 * partials of every masked position, written into the library workspace and not folded
 * into (c, x_hat).  One kernel.  Its use is timing the reduction kernel by itself (a CUDA
 * graph of these calls); arguments and errors as for fdllm_confidence. */
fdllm_status fdllm_vocab_reduce(const void *logits, int dtype, int B, int L, int V,
                                const uint8_t *mask, void *stream);

/* Steps a2-a5 alone (Alg. 1 sort, scan, select, reveal) on given confidences.
 *   conf    [B, L] fp32 device, read at masked positions; a masked value outside (0, 1]
 *           (NaN included) makes the row FDLLM_ROW_NONFINITE.
 *   argmax  [B, L] int32 device, the token revealed at each committed position.
 * mask, param, mode and the outputs as in fdllm_select.  Needs no workspace. */
fdllm_status fdllm_select_from_conf(const float *conf, const int32_t *argmax, int B, int L,
                                    uint8_t *mask, double param, int mode,
                                    int32_t *out_tokens, uint8_t *out_commit, int32_t *out_n,
                                    void *stream);

/* Input movement for the end-to-end path (the paper has no counterpart: it moves data, it
 * computes nothing): copies the rows of the masked positions of `src` [B, L, V] (dtype as
 * given) to the same offsets of `dst`, a device buffer of the same shape; rows of unmasked
 * positions of dst are not written.  src may be device memory or page-locked host memory
 * (cudaHostAlloc / torch pin_memory), which the GPU reads directly over the host link, so
 * that only the masked rows cross it.  mask [B, L] uint8 device.  Pageable host memory is
 * rejected (FDLLM_ERR_ARG); src and dst 16-byte aligned, V * sizeof(dtype) a multiple of 16
 * (FDLLM_ERR_ALIGN).  Asynchronous on `stream`. */
fdllm_status fdllm_gather_masked_rows(const void *src, void *dst, int dtype, int B, int L, int V,
                                      const uint8_t *mask, void *stream);

/* One selection step end to end on host buffers (Alg. 1's step as fdllm_select computes it;
 * this entry only moves data around it): the call a host program makes when its logits
 * are in host memory.  Arguments as in fdllm_select, except:
 *   logits  [B, L, V] in page-locked host memory (cudaHostAlloc / cudaHostRegister / torch
 *           pin_memory): the GPU reads the rows of masked positions over the host link and
 *           nothing else; pageable host memory is copied whole first (slower); device
 *           memory is read in place.  16-byte aligned.
 *   mask, out_tokens, out_commit, out_n  host (or device) arrays of fdllm_select's shapes;
 *           mask is updated in place and out_tokens keeps its values at positions not
 *           committed, as in fdllm_select.
 * The library copies mask and out_tokens to a device staging buffer of its own (per device,
 * grown on demand with cudaMalloc, released by fdllm_release_workspace), runs the step on
 * `stream` with the library workspace, copies out_tokens, out_commit, out_n and the mask
 * back and synchronises `stream` before it returns: the results are in place when the call
 * returns.  Argument errors are reported before anything is enqueued; the same device
 * errors as fdllm_select (fdllm_device_status).  Not for stream capture (it synchronises).
 * Calls share the staging buffer and the library workspace of their device: calls from
 * several host threads at once must be serialised by the caller.  The paper has no
 * counterpart. */
fdllm_status fdllm_select_host(const void *logits, int dtype, int B, int L, int V,
                               uint8_t *mask, double param, int mode, int32_t *out_tokens,
                               uint8_t *out_commit, int32_t *out_n, void *stream);

/* Step a1 fused with the LM head (the projection that produces the logits, Sec. 3
 * "Notation": p_i = softmax of the logits of position i), then steps a2-a5 as in
 * fdllm_select.  For every masked position the logits x = W h are computed on the tensor
 * cores (bf16 inputs, fp32 accumulation) and reduced to (c, x_hat) in the GEMM's epilogue:
 * the B*L*V logits are never written to memory.
 *   hidden   [B, L, H] bf16 device, the final hidden state of each position (read at masked
 *            positions only); 16-byte aligned.
 *   w_vocab  [V, H] bf16 device, the vocabulary projection, row v = the weights of token v;
 *            16-byte aligned.
 *   H        hidden size, a multiple of 8 (16-byte rows); V >= 1, any value.
 * mask, param, mode and the outputs as in fdllm_select (B*L <= FDLLM_MAX_ROWS, L <=
 * FDLLM_MAX_L).  Uses the library-owned workspace (at most B*L*(2H + 16*ceil(V/208) + 12)
 * bytes and a header), allocated outside the step as for fdllm_select.  Asynchronous on
 * `stream`.  The GEMM's tiling (row tiles of 128, CTA pairs, or vocabulary slabs for at most
 * 32 rows) is chosen from B*L and V; the environment variables FDLLM_LMHEAD_GEMM (solo,
 * pair, slab) and FDLLM_LMHEAD_BN (256, 208) force one, for measurements.
 * Results agree with fdllm_select applied to the fp32 logits fdllm_lmhead_logits writes
 * under the same tiling (the same tensor-core accumulation): tokens bit-exact, confidences
 * within 1e-5. */
fdllm_status fdllm_lmhead_select(const void *hidden, const void *w_vocab, int B, int L, int H,
                                 int V, uint8_t *mask, double param, int mode,
                                 int32_t *out_tokens, uint8_t *out_commit, int32_t *out_n,
                                 void *stream);

/* Step a1 alone on the LM head: out_conf (fp32) and out_argmax (int32), [B, L] device, written
 * at masked positions (NaN and -1 for a row whose logits hold a NaN or an infinite maximum).
 * Arguments as fdllm_lmhead_select. */
fdllm_status fdllm_lmhead_confidence(const void *hidden, const void *w_vocab, int B, int L,
                                     int H, int V, const uint8_t *mask, float *out_conf,
                                     int32_t *out_argmax, void *stream);

/* The same tensor-core GEMM with its accumulators stored instead of reduced: out_logits
 * [B, L, V] fp32 device, written at the masked positions' rows only (the unfused path, and
 * the exact inputs against which the fused reduction is checked). */
fdllm_status fdllm_lmhead_logits(const void *hidden, const void *w_vocab, int B, int L, int H,
                                 int V, const uint8_t *mask, float *out_logits, void *stream);

/* Model forward pass used by fdllm_decode_loop.  It must only enqueue stream-ordered GPU
 * work on `stream`: it is called while the loop body is being captured into a CUDA graph
 * (once, or twice when the driver rejects the first capture and the body is captured again
 * without programmatic dependent launches), and the captured work is replayed at every
 * step.  It must not synchronise or allocate.  It writes logits [B, block_len, V]
 * of the current block into `logits` for the rows with block_mask != 0.  loop_state is a
 * device pointer to two int32 values read at run time: [0] the global step (forward passes
 * so far), [1] the current block.  Return 0 on success. */
typedef int (*fdllm_forward_fn)(void *user, const int32_t *loop_state,
                                const uint8_t *block_mask, void *logits, void *stream);

/* Algorithm 1's outer loop on the GPU, with no host round trip per step: for each of
 * gen_len / block_len blocks, start with the block fully masked and repeat {forward pass;
 * selection with (mode, param) as in fdllm_select; reveal} while the block has masked
 * positions (Alg. 1: a block's steps go on until none of its positions is masked), then
 * move to the next block.
 * The loop is one CUDA graph with a conditional WHILE node; the forward pass, the two
 * selection kernels and a controller kernel form its body.
 *   logits          [B, block_len, V] device buffer the forward pass writes (dtype as given).
 *   seq_tokens      [B, gen_len] int32 device output: the committed tokens (-1 if none).
 *   nfe_per_block   [gen_len / block_len] int32 device output: steps (NFE) per block.
 *   max_steps       bound on the total number of steps; reaching it ends the loop early
 *                   and returns FDLLM_ERR_DEVICE.
 * A step whose selection reports a row as FDLLM_ROW_NONFINITE ends the loop after that
 * step with FDLLM_ERR_NONFINITE (such a row commits nothing, so its block would never
 * finish); a step that reports FDLLM_ROW_DEVICE_ERROR ends it with FDLLM_ERR_DEVICE.
 * nfe_per_block then holds the steps of the blocks reached and out_steps the steps taken.
 *   out_steps       host int: total steps taken.
 * Synchronous: returns when the generation is finished.  Allocates its own small buffers
 * and the library workspace (outside the graph).  Limits as fdllm_select with L = block_len;
 * modes FDLLM_PROFILE, FDLLM_FACTOR and FDLLM_THRESHOLD.  Errors: FDLLM_ERR_ARG for a bad
 * argument (checked before any device work) or a forward pass that returned nonzero;
 * FDLLM_ERR_CUDA for a failed graph build or launch.  Uses the library-owned workspace of
 * fdllm_select: no other selection may run on this device from another thread meanwhile.
 * Every step commits at least one position of each row that still has masked positions, so
 * each block ends after at most block_len steps. */
fdllm_status fdllm_decode_loop(int B, int gen_len, int block_len, int V, int dtype,
                               double param, int mode, fdllm_forward_fn forward, void *user,
                               void *logits, int32_t *seq_tokens, int32_t *nfe_per_block,
                               int max_steps, int *out_steps, void *stream);

/* fdllm_decode_loop with the LM head inside the loop body: the forward pass writes the final
 * hidden states [B, block_len, H] bf16 into `hidden` (rows with block_mask != 0), and each
 * step's selection is fdllm_lmhead_select against w_vocab [V, H] bf16 (the logits never
 * reach memory).  Arguments, limits and errors otherwise as fdllm_decode_loop and
 * fdllm_lmhead_select (H a multiple of 8; w_vocab NULL: FDLLM_ERR_ARG). */
fdllm_status fdllm_decode_loop_lmhead(int B, int gen_len, int block_len, int H, int V,
                                      const void *w_vocab, double param, int mode,
                                      fdllm_forward_fn forward, void *user, void *hidden,
                                      int32_t *seq_tokens, int32_t *nfe_per_block, int max_steps,
                                      int *out_steps, void *stream);

/* Heterogeneity-bonus diagnostics (Prop. heterogeneity-bonus, Eq. heterogeneity_decomp,
 * Remark adaptive-factor).  For each batch row, the masked confidences are sorted as the
 * selection sorts them (descending, ties: lower position first); at rank n = 1..m_b:
 *   out_G[b, n-1]     = G_n = max{0, sum_{j<=n} c_(j) - (n-1)} - (1 - c_(n))
 *   out_F[b, n-1]     = F_n = (n+1) c_(n) - n                (factor core)
 *   out_B[b, n-1]     = B_n = sum_{j<n} (c_(j) - c_(n))       (heterogeneity bonus)
 *   out_feff[b, n-1]  = f_eff(n) = 1 - delta + B_n           (Remark adaptive-factor)
 *   out_order[b, n-1] = the position holding c_(n)
 * Ranks n > m_b get NaN (order -1).  G_n = F_n + B_n wherever the lower bound is positive,
 * so the profile rule with margin delta behaves as the factor rule with the effective
 * factor f_eff(n).
 *   conf   [B, L] fp32 device (e.g. from fdllm_confidence), read at masked positions:
 *          values in [0, 1], or NaN (a NaN ranks after every number, so the terms of its
 *          rank and of every later rank are NaN); other values give unspecified terms.
 *   mask   [B, L] uint8 device, nonzero = masked (not modified).
 *   delta  the profile rule's margin (delta = 1 - param of fdllm_select), finite.
 *   out_G, out_F, out_B, out_feff  [B, L] fp64 device, each nullable; out_order [B, L]
 *   int32, nullable.
 * Asynchronous on `stream`; needs no workspace. */
fdllm_status fdllm_profile_terms(const float *conf, const uint8_t *mask, int B, int L,
                                 double delta, double *out_G, double *out_F, double *out_B,
                                 double *out_feff, int32_t *out_order, void *stream);

/* ------------------------------------------------------------ the 4-bit prefix cache --- */
/* The paper's decoding keeps the keys and values of the finished prefix and lets the active
 * block's queries attend to them at every step (PrefixCache, Sec. 5); the cache itself is
 * the model's side of the step, which the paper takes as given.  The entry points below hold
 * such a cache in 4 bits, in pages, for one layer: write (fdllm_cache_append), read back
 * (fdllm_cache_read), attend (fdllm_cache_attention), measure how much attention each key
 * receives (fdllm_cache_key_weights) and drop the keys that receive little
 * (fdllm_cache_evict).  fdllm_qk_norm_rope makes the queries and keys that enter it.  All of
 * them are asynchronous on `stream`, allocate nothing, use no library workspace and may be
 * captured into a CUDA graph (in the forward pass of fdllm_decode_loop, for instance); the first
 * call of each with a head size, dtype and range of lengths sets its kernel up on the device and
 * must come before a capture.  They are forms for inference and have no gradients.
 *
 * A row of D values (one token's keys, or values, of one head) is held as 4-bit codes with
 * two bfloat16 numbers, value = offset + scale * code:
 *   offset = bf16(min), scale = bf16((max - min) / 15),
 *   code   = clamp(rint((x - offset) / scale), 0, 15), 0 when scale is 0,
 * computed in fp32 (bf16(): round to nearest even; rint(): half to even).  A row with a NaN or
 * an infinity, or whose range overflows, is held as NaN (all of its values read as NaN).
 *
 * Pages are found through block_table [B, max_pages] int32 (device): slot j of sequence b is
 * slot j % page_size of page block_table[b][j / page_size].  Slots keep the order of the
 * tokens; attention does not depend on it.  Offsets into the cache are 64-bit.
 */
typedef struct {
    void *k_codes;   /* uint8 [pages, heads, page_size, D/2]: channel 2i in the low half of
                        byte i                                                            */
    void *v_codes;   /* uint8 [pages, heads, D, page_size/2]: slot 2i in the low half of
                        byte i (channel-major, as the attention's products read it)       */
    void *k_affine;  /* bfloat16 [pages, heads, page_size, 2]: (scale, offset)            */
    void *v_affine;  /* bfloat16 [pages, heads, page_size, 2]: (scale, offset)            */
    int pages;
    int heads;       /* key/value heads; pages * heads below 2^31                         */
    int page_size;   /* 32, 64, 128 or 256                                                */
    int head_dim;    /* D: 64 or 128                                                      */
} fdllm_cache;
/* The four arrays are device memory of the caller, 16-byte aligned, of any content before
 * the slots are written (they need not be cleared).  The struct itself is host memory, read
 * during the call.  Every entry point checks it: FDLLM_ERR_ARG for a null pointer or a size
 * out of range, FDLLM_ERR_ALIGN for a base that is not 16-byte aligned. */

/* Per-head RMS norm of queries and keys and their rotary positions in one pass:
 *   y = x / sqrt(mean(x^2) + eps) * weight        (skipped for a tensor whose weight is NULL)
 *   pair p of y turned by the angle positions[axis(p)][t] * inv_freq[p].
 * All arithmetic in fp32, rounded once; the angle is reduced exactly (64-bit fixed point, in
 * turns), so positions up to 2^31 keep their full accuracy.
 *   q, k         [T, Hq, D], [T, Hk, D] in dtype, the channels of a row contiguous;
 *                q_strides / k_strides: {token, head} strides in elements, host (rows of a
 *                packed projection, for instance).  k may be NULL with Hk = 0.
 *   D            2 to 512, even.
 *   q_weight, k_weight  [D] in dtype, or NULL.
 *   positions    [axes, T] int32 device, any sign; axes 1 to 4 (time, height, width, ...).
 *   sections     host, axes ints summing to pairs: the first sections[0] pairs follow axis
 *                0, and so on; NULL with axes = 1.
 *   inv_freq     host, `pairs` finite doubles (radians per position), pairs <= D / 2; channels
 *                from 2 * pairs on are normed but not turned.
 *   interleaved  0: pair p is channels (p, p + pairs); 1: channels (2p, 2p + 1).
 *   out_q, out_k contiguous [T, Hq, D], [T, Hk, D] in dtype; out_q may be q itself where q is
 *                contiguous (likewise k).
 * T = 0 is a no-op.  Errors: FDLLM_ERR_ARG. */
fdllm_status fdllm_qk_norm_rope(const void *q, const int64_t *q_strides, const void *k,
                                const int64_t *k_strides, int dtype, int T, int Hq, int Hk,
                                int D, const void *q_weight, const void *k_weight, double eps,
                                const int32_t *positions, int axes, const int32_t *sections,
                                const double *inv_freq, int pairs, int interleaved, void *out_q,
                                void *out_k, void *stream);

/* Writes n tokens' keys and values into slots start[b] .. start[b] + count[b] - 1.
 *   k, v   [B, n, heads, D] in dtype (bf16, fp16 or fp32), channels contiguous; strides
 *          {batch, token, head} in elements, host; base and strides 16-byte multiples
 *          (FDLLM_ERR_ALIGN).
 *   start  [B] int32 device, or NULL: 0.      count  [B] int32 device, or NULL: n; tokens from
 *          count[b] on are padding and not written.
 * A token whose slot is past the table or in a page out of range is not written, and of a
 * sequence whose start is negative none is (device data, not checked on the host; attention over
 * such a slot reports NaN, and fdllm_cache_read takes each slot for itself).  Two slots
 * share a byte of v_codes: calls writing one sequence must be ordered on the GPU. */
fdllm_status fdllm_cache_append(const fdllm_cache *cache, const int32_t *block_table, int B,
                                int max_pages, const int32_t *start, const int32_t *count,
                                const void *k, const int64_t *k_strides, const void *v,
                                const int64_t *v_strides, int dtype, int n, void *stream);

/* Reads slots start[b] .. start[b] + n - 1 back as dense rows: out_k, out_v contiguous
 * [B, n, heads, D] in dtype (offset + scale * code in fp32, rounded once).  Rows from count[b]
 * on (count NULL: n) are zero; a slot that does not exist reads as NaN.  start, count as in
 * fdllm_cache_append. */
fdllm_status fdllm_cache_read(const fdllm_cache *cache, const int32_t *block_table, int B,
                              int max_pages, const int32_t *start, const int32_t *count,
                              void *out_k, void *out_v, int dtype, int n, void *stream);

/* Attention of Lq queries of each sequence over its cached keys and the block's own:
 *   s_ij = scale * (q_i . k_j),   out_i = sum_j softmax_j(s_ij) v_j,
 *   out_lse_i = log sum_j exp(s_ij).
 * Query head h reads key/value head h / (Hq / heads).
 *   q            [B, Lq, Hq, D] bf16 or fp16, Hq a multiple of the cache's heads; strides
 *                {batch, token, head} in elements, host.
 *   cache_lens   [B] int32 device: slots 0 .. cache_lens[b] - 1 are attended to.
 *   k_new, v_new [B, Ln, heads, D] in q's dtype: the block's own keys and values, not in the
 *                cache, strides as q's; NULL with Ln = 0.
 *   new_lens     [B] int32 device, or NULL: Ln.  Own keys from new_lens[b] on are not seen.
 *   causal       1: query i sees own keys j <= i only (all cached keys always).
 *   out          [B, Lq, Hq, D] in q's dtype, contiguous.   out_lse [B, Lq, Hq] fp32 or NULL.
 *   workspace    device, 256-byte aligned, fdllm_cache_attention_workspace_bytes() bytes, of
 *                any content; calls that may overlap on the GPU need their own, and so do
 *                calls of several host threads on one stream (a call is two launches).
 * A query that sees no key gets out = 0 and out_lse = -inf.  A sequence whose cache_lens or
 * new_lens is out of range (negative, past the table, past Ln) or that meets a page out of
 * range among its first cache_lens slots gets NaN, for all its rows where the lengths are
 * wrong and for the heads and rows that meet the page otherwise.  Non-finite values behind
 * the lengths or the causal bound change nothing, and no query's values, whatever their size, take
 * accuracy from another's results.  Scores and sums are fp32; a weight, with the scale of the
 * cached row folded in, enters the second product as two fp16 numbers, 22 bits of it (own values:
 * two numbers of q's dtype).
 * q, k_new and v_new: 16-byte aligned bases and strides (FDLLM_ERR_ALIGN). */
fdllm_status fdllm_cache_attention(const void *q, const int64_t *q_strides, int dtype, int B,
                                   int Lq, int Hq, const fdllm_cache *cache,
                                   const int32_t *block_table, int max_pages,
                                   const int32_t *cache_lens, const void *k_new,
                                   const int64_t *k_strides, const void *v_new,
                                   const int64_t *v_strides, int Ln, const int32_t *new_lens,
                                   int causal, double scale, void *out, float *out_lse,
                                   void *workspace, size_t workspace_bytes, void *stream);

/* Bytes of workspace fdllm_cache_attention needs for these sizes (a host function; it asks
 * the current device for its number of SMs).  0 for sizes out of range. */
size_t fdllm_cache_attention_workspace_bytes(int B, int Lq, int Hq, int heads, int head_dim);

/* The attention each cached key receives, summed over the queries and the heads that read it:
 *   weights_out[b][h][j] = weights_in[b][h][j] + sum_{i, g} exp(scale * q_ig . k_j - lse_ig)
 * for j < cache_lens[b], and 0 from there to max_len - 1.
 *   q, cache, block_table, cache_lens, scale   as in fdllm_cache_attention.
 *   lse          [B, Lq, Hq] fp32, contiguous: fdllm_cache_attention's out_lse (a row of -inf
 *                counts as 0, whatever its queries hold: it saw no key, or is padding).
 *   weights_in   [B, heads, max_len] fp32 or NULL (0); weights_out the same shape, may be
 *                weights_in.
 * Deterministic (no atomics).  A sequence whose length is negative, past the table or past
 * max_len gets NaN in all its weights, a key in a page out of range NaN in its own. */
fdllm_status fdllm_cache_key_weights(const void *q, const int64_t *q_strides, int dtype, int B,
                                     int Lq, int Hq, const fdllm_cache *cache,
                                     const int32_t *block_table, int max_pages,
                                     const int32_t *cache_lens, const float *lse, double scale,
                                     const float *weights_in, float *weights_out, int max_len,
                                     void *stream);

/* Keeps `budget` keys of each sequence and head: the first keep_first slots, the last
 * keep_last, and of the rest those with the largest weights (equal weights: the lower slot; a
 * NaN weighs less than any number).  The kept rows are copied in slot order into the pages of
 * dst_table [B, dst_max_pages], slots 0, 1, ...; each head keeps its own set.  A sequence of
 * at most `budget` slots keeps all of them.
 *   weights      [B, heads, max_len] fp32 (fdllm_cache_key_weights).
 *   out_lens     [B] int32: min(cache_lens[b], budget); -1 for a sequence whose length is
 *                negative, past the table or past max_len (nothing else is written for it but
 *                the padding).
 *   out_weights  [B, heads, budget] fp32: the kept keys' weights, 0 behind out_lens.
 *   out_index    [B, heads, budget] int32: the slots they came from, -1 behind out_lens.
 * The source is not modified; dst_table's pages must not be among the source's, and
 * dst_max_pages * page_size >= budget (FDLLM_ERR_ARG).  Rows whose source or destination page
 * is out of range are not copied.  budget >= 1, keep_first + keep_last <= budget. */
fdllm_status fdllm_cache_evict(const fdllm_cache *cache, const int32_t *block_table, int B,
                               int max_pages, const int32_t *cache_lens, const float *weights,
                               int max_len, int budget, int keep_first, int keep_last,
                               const int32_t *dst_table, int dst_max_pages, int32_t *out_lens,
                               float *out_weights, int32_t *out_index, void *stream);

/* ------------------------------------------------------ drafting and its verification --- */
/* A drafter proposes tokens and a target model takes or rejects them: a chain of them, or a tree
 * whose branches are alternatives.  Nodes of a draft: node 0 is the root, the last committed token
 * (the token whose keys are not in the cache yet); nodes 1 .. M - 1 are drafted tokens, each
 * behind its parent, parents[b][j] < j.  fdllm_tree_mask and fdllm_cache_tree_attention run the
 * nodes through the target in one pass, fdllm_verify_draft takes the tokens, and
 * fdllm_distill_loss, fdllm_distill_grad and fdllm_distill_step train the drafter on its target's top
 * logits.  All of them are asynchronous on `stream`, allocate nothing and may be captured into a
 * CUDA graph; the first call of each with a dtype (attention: with a head size, dtype and range of
 * lengths) on a device sets its kernels up and must come before a capture.  They are
 * deterministic: the same inputs give the same bits. */

/* The bits of which node sees which, and the nodes' depths.
 *   parents    [B, M] int32 device; node 0's is not read.  A node whose parent is not in 0 .. j - 1
 *              is detached: a root of its own.
 *   lens       [B] int32 device, or NULL: M.  Nodes from lens[b] on are padding (a value out of
 *              0 .. M counts as the nearer end).
 *   M          1 to FDLLM_MAX_L.
 *   out_mask   [B, M, ceil(M / 32)] uint32: bit j % 32 of word j / 32 of row i is set where node j is
 *              node i or an ancestor of it.  Padding rows are 0.
 *   out_depth  [B, M] int32, or NULL: steps from the root (a node's position is the root's plus its
 *              depth); -1 for padding. */
fdllm_status fdllm_tree_mask(const int32_t *parents, const int32_t *lens, int B, int M,
                             uint32_t *out_mask, int32_t *out_depth, void *stream);

/* fdllm_cache_attention with a bit for each query and own key in causal's place: query i sees all
 * cached keys and the own keys j whose bits are set.
 *   mask   [B, Lq, ceil(Ln / 32)] uint32 device, bit j % 32 of word j / 32 of row i (fdllm_tree_mask's
 *          out_mask for Lq = Ln = M; any other pattern does as well, an empty row among them).  Bits
 *          from new_lens[b] on are not read as set.  May be NULL where Ln = 0.
 * Everything else, the workspace and its size among it, as fdllm_cache_attention; a non-finite
 * value of an own key reaches the queries that see it and no others. */
fdllm_status fdllm_cache_tree_attention(const void *q, const int64_t *q_strides, int dtype, int B,
                                        int Lq, int Hq, const fdllm_cache *cache,
                                        const int32_t *block_table, int max_pages,
                                        const int32_t *cache_lens, const void *k_new,
                                        const int64_t *k_strides, const void *v_new,
                                        const int64_t *v_strides, int Ln, const int32_t *new_lens,
                                        const uint32_t *mask, double scale, void *out,
                                        float *out_lse, void *workspace, size_t workspace_bytes,
                                        void *stream);

/* Bytes of workspace fdllm_verify_draft needs (a pure host function).  0 for sizes out of range. */
size_t fdllm_verify_draft_workspace_bytes(int B, int M, int V, int dtype);

/* Takes drafted tokens by the target's probabilities and given random numbers, so that what
 * comes out is distributed as the target's own samples.  With p_c = softmax(target row c /
 * temperature), q_c = softmax(draft row c / draft_temperature), from the root on:
 *   draft given (a chain drawn from q): node c + 1, token d, is taken iff
 *       uniform[b][c + 1] * q_c(d) < p_c(d).
 *       Behind the first that is not, the next token is drawn from max(p_c - q_c, 0).
 *   draft NULL (tokens that were chosen, not drawn; a chain or a tree): the children of c are
 *       tried in order of their numbers, child k iff uniform[b][k] * (1 - S) < p_c(d_k) with S the
 *       p_c of the children tried before it (a token tried before counts 0).  Where none is
 *       taken, the next token is drawn from p_c without the tokens tried.
 *   temperature 0 (greedy): a child is taken iff its token is the argmax after c (lowest index on
 *       ties); the next token is the argmax.
 *   A token is drawn as argmax_v r(v) / noise[b][v] (lowest index on ties) from the weights r: noise
 *   holds exponential variables.  Weights that are all 0 give way to p_c, and where no token
 *   can be drawn from that either, the next token is the argmax.
 * Probabilities and weights are fp32 (relative error within 1e-5), the tests of tokens 64-bit
 * products of them.
 * Rows that are not on the way change nothing; of large trees they are not read.
 *   target     [B, M, V] device, dtype as given, row j the logits after node j; V any from 1 to 2^20,
 *              the values of a row contiguous, rows anywhere (FDLLM_ERR_ALIGN: a base that is not a
 *              multiple of the value's size); target_strides {batch, row} in elements, host.
 *   draft      [B, M - 1, V] in the same dtype, row j the logits that node j + 1 was drawn from, strides
 *              as target's; or NULL.  Only with parents NULL and temperature > 0 (FDLLM_ERR_ARG).
 *   tokens     [B, M] int32 device: the nodes' tokens (node 0's is not read).  A token out of the
 *              vocabulary is never taken.
 *   parents    [B, M] int32 device, or NULL: a chain.  A node whose parent is not in 0 .. j - 1 is
 *              never reached.
 *   lens       [B] int32 device, or NULL: M.  Nodes from lens[b] on are padding, their rows not
 *              read (a value out of 1 .. M counts as the nearer end).
 *   M          1 (no drafts: the next token is drawn from row 0) to FDLLM_MAX_L.
 *   temperature, draft_temperature   1e-6 to 1e6, or temperature 0.
 *   uniform    [B, M] fp32 device in [0, 1); entry 0 is not read.   noise  [B, V] fp32 device, > 0; a
 *              token whose noise is NaN, negative or infinite is not drawn.  Both may be NULL where
 *              temperature is 0.
 *   out_tokens [B, M] int32: the taken tokens, then the next token; -1 behind.
 *   out_nodes  [B, M] int32: the root (0), then the taken nodes: the rows whose keys and values
 *              enter the cache; -1 behind.
 *   out_n      [B] int32: taken tokens, 0 .. M - 1; FDLLM_ROW_NONFINITE (and -1 in the row of the
 *              others) where a row on the way holds a NaN or its maximum is infinite;
 *              FDLLM_ROW_DEVICE_ERROR where a kernel of this call gave up a bounded wait, or one of
 *              another call did and fdllm_cache_status was not asked since.
 *   workspace  device, 256-byte aligned, fdllm_verify_draft_workspace_bytes() bytes of any content;
 *              calls that may overlap on the GPU need their own. */
fdllm_status fdllm_verify_draft(const void *target, const int64_t *target_strides,
                                const void *draft, const int64_t *draft_strides, int dtype, int B,
                                int M, int V, const int32_t *tokens, const int32_t *parents,
                                const int32_t *lens, double temperature, double draft_temperature,
                                const float *uniform, const float *noise, int32_t *out_tokens,
                                int32_t *out_nodes, int32_t *out_n, void *workspace,
                                size_t workspace_bytes, void *stream);

/* The loss of a student on its teacher's top logits at the masked positions.  With
 * q = softmax(x / temperature) of a position's logits x, and of its listed tokens the teacher's
 * probabilities p_k:
 *   teacher_lse NULL: p = softmax(top_logits / temperature) over the listed tokens, R = 0;
 *   teacher_lse given: p_k = exp(top_logits_k / temperature - teacher_lse), and R = max(0, 1 - sum p)
 *       is the teacher's rest, held against the student's rest r = sum of q over all other tokens:
 *   out_loss = sum_k p_k (log p_k - log q_k) + R (log R - log r).
 * A term with p_k = 0, or R = 0, is 0, and so is the rest's where the student has no other token
 * (r = 0).  All in fp32, sums of exponentials relative to their own maxima, r summed by itself.
 *   logits       [B, L, V] device, dtype as given, base 16-byte aligned (FDLLM_ERR_ALIGN), V any
 *                from 1 to 2^20; B * L below 2^31.  Read at masked positions only.
 *   mask         [B, L] uint8 device, nonzero = masked (counted).
 *   top_index    [B, L, K] int32 device: the listed tokens; an index out of 0 .. V - 1 is an absent
 *                entry; masses of a token listed more than once add up.   K  1 to 1024.
 *   top_logits   [B, L, K] device in top_dtype (bf16, fp16 or fp32).
 *   teacher_lse  [B, L] fp32 device: logsumexp(all the teacher's logits / temperature); or NULL.
 *   temperature  1e-6 to 1e6.
 *   out_loss     [B, L] fp32: 0 at positions that are not masked; NaN where a masked row of the
 *                student holds a NaN or its maximum is infinite, or the teacher's numbers are NaN.
 *   out_stats    [B, L, 4] fp32, 16-byte aligned, or NULL: what fdllm_distill_grad needs. */
fdllm_status fdllm_distill_loss(const void *logits, int dtype, int B, int L, int V,
                                const uint8_t *mask, const int32_t *top_index,
                                const void *top_logits, int top_dtype, int K,
                                const float *teacher_lse, double temperature, float *out_loss,
                                float *out_stats, void *stream);

/* Its gradient, given that of each position's loss:
 *   out_grad = grad_loss / temperature * (q_v (P + R) - p_v)     at a listed token, P = sum p,
 *              grad_loss / temperature * (q_v (P + R) - R q_v / r)  at another,
 * 0 at positions that are not masked, in the logits' dtype (rounded once), NaN where the loss is.
 *   stats      fdllm_distill_loss's out_stats for the same arguments.
 *   grad_loss  [B, L] fp32 device, read at masked positions.
 *   out_grad   [B, L, V], 16-byte aligned; may be `logits` itself. */
fdllm_status fdllm_distill_grad(const void *logits, int dtype, int B, int L, int V,
                                const uint8_t *mask, const int32_t *top_index,
                                const void *top_logits, int top_dtype, int K,
                                const float *teacher_lse, double temperature, const float *stats,
                                const float *grad_loss, void *out_grad, void *stream);

/* Both in one call that reads the logits once, where grad_loss is known beforehand (1 / count, for a
 * mean).  Arguments as above. */
fdllm_status fdllm_distill_step(const void *logits, int dtype, int B, int L, int V,
                                const uint8_t *mask, const int32_t *top_index,
                                const void *top_logits, int top_dtype, int K,
                                const float *teacher_lse, double temperature,
                                const float *grad_loss, float *out_loss, void *out_grad,
                                void *stream);

/* The sticky device error of fdllm_cache_attention, fdllm_cache_tree_attention,
 * fdllm_cache_key_weights, fdllm_verify_draft and the distillation calls on the current device:
 * synchronises `stream`, returns FDLLM_ERR_DEVICE if one of their kernels gave up a bounded wait since
 * the last call (the results of the calls since then are unusable; fdllm_verify_draft reports
 * FDLLM_ROW_DEVICE_ERROR for every sequence until then), FDLLM_OK otherwise, and clears it.  The
 * word is the device's, whichever thread's call it was: who asks, asks for all. */
fdllm_status fdllm_cache_status(void *stream);

/* Health check of those kernels' bounded waits: enqueues a warp that waits on a barrier nobody
 * completes and gives up after `tries` tries (1 to 2^18; 0: the kernels' own limit, about a
 * second), so that fdllm_cache_status reports FDLLM_ERR_DEVICE once. */
fdllm_status fdllm_cache_check_wait(int tries, void *stream);

/* Health check of the library's failure detection: every wait inside the kernels is
 * bounded, and a wait that runs out records a device error and lets the kernel return
 * instead of hanging.  This launches one thread that waits on a barrier nobody completes,
 * with a limit of `seconds` (0 < seconds <= 10), synchronises `stream` and returns
 * FDLLM_ERR_DEVICE when the wait ran out and was reported as it should (FDLLM_OK would mean
 * the wait did not run out).  The device stays usable afterwards.  The paper has no
 * counterpart. */
fdllm_status fdllm_check_bounded_wait(double seconds, void *stream);

/* Synchronises `stream`, then reports (and clears) the sticky device error of the library
 * workspace on the current device: FDLLM_ERR_DEVICE if a kernel gave up a bounded wait
 * since the last call, else FDLLM_ERR_NONFINITE if a selection since the last call found a
 * row of FDLLM_ROW_NONFINITE, FDLLM_OK otherwise.  For fdllm_select_ws, pass the workspace to
 * fdllm_workspace_status instead.  Clearing an error also resets the workspace's work
 * counter, which a launch that gave up may have left mid-queue, so that the next call
 * starts from a clean header. */
fdllm_status fdllm_device_status(void *stream);
fdllm_status fdllm_workspace_status(void *workspace, void *stream);

/* Frees the library workspace of the current device (synchronises the device). */
void fdllm_release_workspace(void);

/* A static English description of a status code. */
const char *fdllm_status_string(int status);

/* Library version, major * 10000 + minor * 100 + patch. */
int fdllm_version(void);

#ifdef __cplusplus
}
#endif

#endif /* FDLLM_H */
