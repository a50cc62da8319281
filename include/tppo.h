/*
 * tppo.h -- C ABI of the B200 (sm_100a) T-PPO token-selective update library.
 *
 * The library computes the part of a Truncated-PPO training step that the paper's method changes:
 * EGAE advantages over possibly truncated responses (Section 3.1, Eq. 6), the policy / value
 * token filter (Section 3.2), and the two losses restricted to the surviving tokens (Eq. 1 and
 * Eq. 4-5; the advantage, policy and value steps of Algorithm 1).  Beside it stand the dense operators
 * of the block around the LM-head: layer norm, linear with a fused epilogue, orthogonalised update.
 *
 * Conventions that hold for every entry point
 *   - Every array pointer is a DEVICE pointer unless the comment says "host".  The caller owns all
 *     buffers, the workspace included; the library allocates nothing and keeps no state between
 *     calls -- with one exception, tppo_egae_static, which works in a device array compiled into
 *     the library and remembers that array's address per device (see there).  Scalars are passed
 *     by value.
 *   - `stream` is a cudaStream_t passed as void*.  Calls enqueue work and return; they never
 *     synchronise the stream or the device.
 *   - Return value: a tppo_status.  Anything the host can detect (null pointer, negative size,
 *     workspace too small, misalignment, unsupported shape) is reported before any kernel is
 *     launched and leaves all outputs untouched.  Problems only the device can see (a target id
 *     outside [0,V), an index outside its array, a scan wait that ran out, a NaN or infinity in
 *     an input) set bits of a status word in the call's output and the affected outputs are
 *     written as 0 -- never NaN, never a trap.
 *   - Packed token layout: sequence i occupies positions [seq_begin[i], seq_begin[i+1]) laid out
 *     prompt | response tokens of earlier windows | response tokens of this window.
 *   - Workspace: query tppo_workspace_bytes() with the same sizes, pass at least that many bytes,
 *     256-byte aligned.  Contents need no initialisation and are garbage afterwards.  Two calls
 *     that may overlap on the GPU need different workspaces.
 */
#ifndef TPPO_H
#define TPPO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    TPPO_OK = 0,
    TPPO_ERR_INVALID_ARG = 1, /* null / negative / inconsistent argument, bad alignment      */
    TPPO_ERR_WORKSPACE = 2,   /* workspace pointer null, misaligned or smaller than required */
    TPPO_ERR_UNSUPPORTED = 3, /* valid request this library cannot serve                     */
    TPPO_ERR_CUDA = 4,        /* a CUDA runtime call failed (launch error, wrong device)     */
    TPPO_ERR_TOO_LARGE = 5    /* problem exceeds a fixed built-in capacity (see *_static)    */
} tppo_status;

/* bits of the device status word */
enum {
    TPPO_DEV_BAD_TARGET = 1,  /* targets[row] outside [0, V): that row contributes nothing   */
    TPPO_DEV_WAIT_TIMEOUT = 2,/* a bounded look-back wait gave up: outputs incomplete        */
    TPPO_DEV_BAD_INDEX = 4,   /* a row / token index outside its array: entry skipped        */
    TPPO_DEV_BAD_SEGMENT = 8, /* segment bounds outside [0, N] or not ascending: skipped     */
    TPPO_DEV_OVERFLOW = 16,   /* an output buffer was too small: the excess was not written  */
    TPPO_DEV_NONFINITE = 32   /* a NaN or infinity was met in an input: see each entry point */
};

typedef enum {
    TPPO_OP_EGAE = 0,
    TPPO_OP_SELECT_TOKENS = 1,
    TPPO_OP_POLICY_LOSS = 2,
    TPPO_OP_VALUE_LOSS = 3,
    TPPO_OP_LMHEAD = 4,
    TPPO_OP_LAYER_NORM = 5, /* N = rows, V = columns                                         */
    TPPO_OP_LINEAR = 6,     /* N = rows M, B = K, V = N of the product; see tppo_linear_fwd  */
    TPPO_OP_MUON = 7,       /* N = rows, V = columns of the matrix                           */
    TPPO_OP_RESIDUAL_NORM = 8, /* N = rows, V = columns                                      */
    TPPO_OP_GRAD_NORM = 9   /* N = number of tensors                                         */
} tppo_op;

/* element types */
enum { TPPO_BF16 = 0, TPPO_F32 = 1 };

/* where the gradient with respect to the logits goes */
enum {
    TPPO_DLOGITS_NONE = 0,    /* forward only (e.g. the old-policy log-probs of Algorithm 1)  */
    TPPO_DLOGITS_FULL = 1,    /* [R, ld] like the logits; rows that are not selected are     */
                              /* zero-filled; may be the logits buffer itself (in place)     */
    TPPO_DLOGITS_COMPACT = 2  /* [n_max, V] dense, row j belongs to the j-th selected row    */
};

/* Library version (major*10000 + minor*100 + patch). Host call. */
int tppo_version(void);

/* Human-readable name of a status code (static string, host). */
const char *tppo_status_string(int status);

/*
 * For tests of the give-up paths of the two kernels that wait on other thread blocks (the scan of
 * tppo_egae and the compaction of tppo_select_tokens, both decoupled look-back chains).  Host call;
 * it changes a process-wide setting that later calls of those two entry points read:
 *   lookback_polls  >= 0: a look-back gives up after this many failed polls of a round of tiles
 *                   (normally about four million); < 0 restores the normal limit
 *   no_publish      != 0: tiles do not publish their partial results, so that every look-back that
 *                   has to wait runs into the limit -- deterministically, without any fault
 * A call made under these settings returns normally with TPPO_DEV_WAIT_TIMEOUT set; its outputs are
 * incomplete but finite and in bounds.  tppo_test_hooks(-1, 0) restores normal operation.
 */
void tppo_test_hooks(int32_t lookback_polls, int32_t no_publish);

/*
 * Workspace bytes needed by one call of `op`.  N = packed tokens, B = sequences / segments,
 * n_max = capacity of the selected-token list, V = vocabulary (0 where it does not apply); the dense
 * operators say at each entry point what the four stand for.
 * Returns 0 for an unknown op.  Host call, launches nothing.
 */
size_t tppo_workspace_bytes(int op, int64_t N, int32_t B, int64_t n_max, int32_t V);

/*
 * EGAE advantages and Monte-Carlo returns (Section 3.1, Eq. 6 with the TD residual of Eq. 3;
 * R_t as defined after Eq. 5; the advantage step of Algorithm 1).
 *
 * For each response segment [seg_begin[i], seg_end[i]) of the packed arrays, backwards in t:
 *     delta_t = rewards[t] + gamma * V(s_{t+1}) - values[t]
 *     A_t     = delta_t + gamma*lambda * A_{t+1},   A_end = 0
 *     R_t     = rewards[t] + gamma * R_{t+1},       R_end = 0
 * where V(s_{t+1}) = values[t+1] inside the segment and, after the last token, 0 if the response
 * finished, else bootstrap[i] -- or, when bootstrap is NULL, values[seg_end[i]-1], the paper's
 * assumption V(s_l) = V(s_{l-1}) for a response cut at the window length l.
 *
 *   rewards, values  [N] fp32      seg_begin, seg_end  [B] int32, ascending, disjoint,
 *   truncated        [B] u8                            0 <= begin <= end <= N (empty allowed)
 *   bootstrap        [B] fp32 or NULL
 *   advantages       [N] fp32 out; returns [N] fp32 out or NULL.  Positions outside every
 *                    segment are written 0.
 *   status           [1] int32 out: device status bits (0 = clean).
 * A reward, value or used bootstrap value inside a segment that is a NaN or an infinity is read as
 * 0 and raises TPPO_DEV_NONFINITE, so the outputs stay finite.
 * Precision: the advantage is carried as G_t = A_t + values[t] (G_t = rewards[t] + gamma*(1-lambda)*
 * V(s_{t+1}) + gamma*lambda*G_{t+1}, so successive values never cancel).  Everything carried across
 * runs of 16 consecutive positions, warps and tiles is fp64 (the composite map of each run
 * included); inside a run the results are evaluated in fp32 from the entering value rounded once.
 * The error of a result is that rounding plus at most 16 fp32 roundings at the magnitude of |G| or
 * |R| inside its run; it does not grow with the length of a response.  N < 2^31.
 * Arrays that are 16-byte aligned take the fast path (TMA copies); others are still handled.
 * The first call in a process looks up the driver's tensor-map encoder (without it every tile takes
 * the slower plain-load path; no error).
 */
int tppo_egae(const float *rewards, const float *values,
              const int32_t *seg_begin, const int32_t *seg_end,
              const uint8_t *truncated, const float *bootstrap,
              int32_t B, int64_t N, float gamma, float lambda,
              float *advantages, float *returns, int32_t *status,
              void *workspace, size_t workspace_bytes, void *stream);

/*
 * tppo_egae without a caller workspace and without any allocation.  (The paper has no counterpart:
 * this is a packaging variant of tppo_egae, same arithmetic, same outputs.)
 *
 * Who needs it: code that runs where device memory cannot be requested -- a plug-in inside a
 * training or serving runtime that has already reserved the whole device for its own pool (a raw
 * cudaMalloc there fails or fragments the pool), or a latency-critical section that must not pay
 * cudaMalloc's device-wide synchronisation -- and that has no spare buffer of its own to lend as
 * workspace.  The scan's tile descriptors live in a fixed array compiled into the library
 * (TPPO_EGAE_STATIC_MAX_TOKENS / 2048 descriptors of 64 bytes plus one counter, about 128 KB); every
 * GPU that loads the library holds that array until the process exits.
 *
 * Arguments and results are those of tppo_egae minus the workspace pair.  Differences:
 *   - N > TPPO_EGAE_STATIC_MAX_TOKENS returns TPPO_ERR_TOO_LARGE before anything is launched.
 *   - The first call on each device looks up the device address of the built-in array (the device
 *     must be current, as for every call) and caches it; make that first call outside any stream
 *     capture.  Later calls only enqueue a clear of the array and the kernel.  The cached address
 *     belongs to the device's current context: after cudaDeviceReset it is stale, and the entry
 *     point must not be used again in that process.
 *   - All calls on a device share the one array, which still holds the previous call's contents:
 *     each call clears it on `stream` before the scan.  Two calls that can overlap on the GPU
 *     (different streams without an ordering between them) race on it and give undefined results;
 *     order them, or use tppo_egae with separate workspaces.
 * The function calls no cudaMalloc / cudaFree and no allocating library routine.
 */
#define TPPO_EGAE_STATIC_MAX_TOKENS 4194304
int tppo_egae_static(const float *rewards, const float *values,
                     const int32_t *seg_begin, const int32_t *seg_end,
                     const uint8_t *truncated, const float *bootstrap,
                     int32_t B, int64_t N, float gamma, float lambda,
                     float *advantages, float *returns, int32_t *status, void *stream);

/*
 * Token filter and compaction (Section 3.2; "selective filtering of prompt and truncated tokens").
 * With o = p - seq_begin[i] for the sequence i that holds position p:
 *   policy token  iff  prompt_len[i]+prev_len[i] <= o < prompt_len[i]+prev_len[i]+new_len[i]
 *                                                       - (truncated[i] ? drop_i : 0)
 *                      (response tokens generated in the current step, finished or not, minus
 *                      the last drop_i tokens of an unfinished sequence; drop_i = tail_drop_seq[i]
 *                      when that array is given, else tail_drop: the paper leaves the number of
 *                      excluded latest tokens open, so it is a parameter, per call or per sequence)
 *   value token   iff  !truncated[i] and prompt_len[i] <= o < prompt_len[i]+prev_len[i]+new_len[i]
 *                      (all generated tokens of finished sequences)
 * each ANDed with the optional byte masks (non-zero = keep).  Prompt tokens are in neither set.
 *
 *   seq_begin [B+1] int32 ascending; prompt_len, prev_len, new_len [B] int32 >= 0; truncated [B] u8
 *   tail_drop >= 0; tail_drop_seq [B] int32 or NULL (a negative entry is read as 0 and raises
 *   TPPO_DEV_BAD_INDEX)
 *   extra_policy_mask, extra_value_mask  [N] u8 or NULL
 *   policy_idx, value_idx  [N] int32 out: selected positions in ascending order (bit-exact,
 *                          run-to-run deterministic); entries past the count are untouched
 *   counts   [4] int32 out: n_policy, n_value, device status bits, 0
 * The counts stay on the device so that the loss calls can consume them without a host round trip.
 */
int tppo_select_tokens(const int32_t *seq_begin, const int32_t *prompt_len,
                       const int32_t *prev_len, const int32_t *new_len,
                       const uint8_t *truncated, int32_t tail_drop, const int32_t *tail_drop_seq,
                       const uint8_t *extra_policy_mask, const uint8_t *extra_value_mask,
                       int32_t B, int64_t N,
                       int32_t *policy_idx, int32_t *value_idx, int32_t *counts,
                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * Fused per-token log-softmax gather + clipped PPO surrogate, forward and backward to the logits
 * (Eq. 1 with decoupled eps_low / eps_high; token-level mean and no KL term per Section 4.1.1;
 * the policy update of Algorithm 1).  For the j-th selected row r = rows[j] (j < n), a = aux_idx[j]:
 *     logp_j = x[r, y] - log sum_v exp(x[r, v]),            y = targets[r]
 *     rho    = exp(logp_j - old_logp[a])
 *     l_j    = -min(rho*adv[a], clip(rho, 1-eps_low, 1+eps_high)*adv[a])
 *     loss   = (1/denom) * sum_j l_j
 *     dlogits[., v] = (adv[a]*rho*active/denom) * (softmax_v - 1[v == y])
 * with active = 0 exactly when the clipped term is strictly the smaller one (the gradient is then
 * zero), and n = min(*n_sel, n_max).  Each selected logits row is read once from HBM.
 *
 *   logits    [R, ld] elements of logits_dtype (TPPO_BF16 or TPPO_F32), row stride ld >= V
 *   targets   [R] int32: the token scored by logits row r (the caller applies the next-token shift)
 *   rows      [n_max] int32 distinct row indices, or NULL for 0..n_max-1
 *   n_sel     [1] int32 device count (e.g. counts+0 of tppo_select_tokens) or NULL for n_max
 *   aux_idx   [n_max] int32 index into old_logp / adv, or NULL to use the row index
 *   old_logp, adv   fp32, length aux_len (bounds-checked against it)
 *   denom     > 0: divisor of the mean (gradient accumulation / several GPUs); <= 0: n
 *   logp, token_loss  [n_max] fp32 out, compact, either may be NULL
 *   loss      [1] fp32 out
 *   stats     [4] int32 out: n, rows clipped at the lower edge, at the upper edge, status bits
 *   dlogits   per dlogits_mode (same element type as the logits); FULL mode may alias `logits`
 *   kernel_hint  0 = choose automatically; other values select a specific kernel for tuning and
 *                testing and never change the result beyond rounding (see tppo_policy_kernels)
 * Zero selected rows give loss 0 and no gradient writes beyond FULL mode's zero fill.
 * Reductions are done in a fixed order: results are run-to-run identical.
 * Range: exp(x - max) is formed from the difference, so finite logits of any magnitude are handled,
 * and -inf logits (a masked vocabulary entry) count as probability 0.  A selected row that holds a
 * NaN or +inf, or nothing but -inf, has no log-softmax: it contributes nothing (logp, loss term and
 * gradient row 0) and raises TPPO_DEV_NONFINITE.
 */
int tppo_policy_loss_fwd_bwd(const void *logits, int32_t logits_dtype,
                             int64_t R, int32_t V, int64_t ld,
                             const int32_t *targets,
                             const int32_t *rows, const int32_t *n_sel, int64_t n_max,
                             const int32_t *aux_idx,
                             const float *old_logp, const float *adv, int64_t aux_len,
                             float eps_low, float eps_high, float denom,
                             float *logp, float *token_loss, float *loss, int32_t *stats,
                             void *dlogits, int32_t dlogits_mode, int32_t kernel_hint,
                             void *workspace, size_t workspace_bytes, void *stream);

/*
 * Forward-only sweep with statistics: the log-probs of the old-policy snapshot (the step of
 * Algorithm 1 that sets pi_theta_old before the updates; the same gather as above, one read of each
 * selected row, no gradient) together with two diagnostics taken from the same pass.  For the j-th
 * selected row r = rows[j] (j < n = min(*n_sel, n_max)), a = aux_idx[j]:
 *     logp[j]    = x[r, y] - log sum_v exp(x[r, v]),          y = targets[r]
 *     entropy[j] = - sum_v p_v log p_v,  p = softmax(x[r, :])  (an entry of probability 0 adds 0)
 *     means[0]   = (1/n) sum_j entropy[j]
 *     means[1]   = (1/n) sum_j (old_logp[a] - logp[j])         (sample estimate of KL(pi_old || pi))
 *   logits, targets, rows, n_sel, n_max, aux_idx, aux_len: as in tppo_policy_loss_fwd_bwd
 *   old_logp   fp32 [aux_len] or NULL (means[1] is then 0 and aux_idx is not used)
 *   logp       [n_max] fp32 out;  entropy [n_max] fp32 out or NULL;  means [2] fp32 out
 *   stats      [4] int32 out: n, 0, 0, status bits
 *   workspace  tppo_workspace_bytes(TPPO_OP_POLICY_LOSS, R, 0, n_max, V) bytes
 * A row with a bad index or target, or whose logits hold a NaN or +inf (or nothing but -inf), gets
 * logp = entropy = 0, is left out of both sums (n still divides) and raises its status bit.
 * Fixed-order reductions: run-to-run identical.
 */
int tppo_policy_logprob_stats(const void *logits, int32_t logits_dtype,
                              int64_t R, int32_t V, int64_t ld,
                              const int32_t *targets,
                              const int32_t *rows, const int32_t *n_sel, int64_t n_max,
                              const int32_t *aux_idx, const float *old_logp, int64_t aux_len,
                              float *logp, float *entropy, float *means, int32_t *stats,
                              void *workspace, size_t workspace_bytes, void *stream);

/* kernel_hint values of tppo_policy_loss_fwd_bwd */
enum {
    TPPO_POLICY_AUTO = 0,
    TPPO_POLICY_TWO_PASS = 1,     /* any shape / dtype: row read twice from global memory      */
    TPPO_POLICY_CLUSTER_SMEM = 2  /* bf16, V % 8 == 0, 16-byte aligned rows: row held in the    */
                                  /* shared memory of a thread-block cluster, read once         */
};

/*
 * Clipped value regression on the value tokens, forward and backward (Eq. 4-5; the value update
 * of Algorithm 1).  For p = value_idx[j], j < n = min(*n_sel, n_max):
 *     Vc = clip(values[p], old_values[p] - xi_low, old_values[p] + xi_high)
 *     l  = 1/2 * max((values[p]-returns[p])^2, (Vc-returns[p])^2),   loss = (1/denom) sum l
 *     dvalues[p] = (values[p]-returns[p])/denom  if the unclipped term is the max (ties included),
 *                  else (Vc-returns[p])/denom if Vc == values[p], else 0
 *   values, old_values, returns [N] fp32; value_idx [n_max] int32 (distinct) or NULL for 0..n_max-1
 *   loss [1] fp32 out; dvalues [N] fp32 out (zero off the value tokens) or NULL
 *   stats [2] int32 out: n, status bits
 * A value token whose value, old value or return is a NaN or an infinity contributes nothing (loss
 * term and gradient 0) and raises TPPO_DEV_NONFINITE.
 */
int tppo_value_loss(const float *values, const float *old_values, const float *returns,
                    int64_t N, const int32_t *value_idx, const int32_t *n_sel, int64_t n_max,
                    float xi_low, float xi_high, float denom,
                    float *loss, float *dvalues, int32_t *stats,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * LM-head variant of the fused policy loss (Eq. 1 as in tppo_policy_loss_fwd_bwd, every one of the
 * M rows selected): the logits x = hidden * weight are a dense [M,K] x [K,V] bf16 contraction on
 * the tensor cores (fp32 accumulation) and are never written to memory.  Outputs are the loss, the
 * per-row log-probs and losses, and the gradients
 *     dhidden = dX * weight^T,   dweight = hidden^T * dX,   dX = (adv*rho*active/denom)(softmax - onehot).
 * The vocabulary is swept twice (statistics, then gradients with the logits recomputed); dX exists
 * only as a bf16 buffer for one chunk of vocabulary columns at a time inside the workspace.
 *
 *   hidden   [M, K] bf16 row-major     weight  [K, V] bf16 row-major     (16-byte aligned)
 *   targets  [M] int32                 aux_idx [M] int32 index into old_logp / adv, or NULL (= row)
 *   old_logp, adv   fp32, length aux_len
 *   logp, token_loss [M] fp32 out or NULL;  loss [1] fp32 out;  stats [4] int32 out as in
 *   tppo_policy_loss_fwd_bwd (n = M)
 *   dhidden  [M, K] bf16 out or NULL;  dweight [K, V] bf16 out or NULL (both NULL: forward only)
 *   chunk_tiles  0 = choose automatically; otherwise the number of 256-column vocabulary tiles per
 *                chunk (low 16 bits), clamped to the automatic choice (which sizes the workspace).
 *                Adding 65536 selects the CTA-pair (cta_group::2) GEMM kernels instead of the single-CTA ones.  For
 *                tuning and testing; changes the result only by the rounding order of dhidden's sum.
 *   workspace    tppo_workspace_bytes(TPPO_OP_LMHEAD, M, K, 0, V) bytes
 * K and V must be multiples of 8 (TPPO_ERR_UNSUPPORTED otherwise).  A row with a target outside
 * [0, V) or an aux index outside [0, aux_len) contributes nothing and raises the status bit.
 * Range: the logits are fp32 sums of K bf16 products and their exponentials are formed as
 * 2^(x*log2(e) - lse*log2(e)), so |x| must stay below 2.3e38 (FLT_MAX / log2 e).  A row whose logits
 * are not finite (a NaN or infinity in its hidden state or in the weight) contributes nothing to
 * the loss and to dweight, gets a zero dX, and raises TPPO_DEV_NONFINITE; dhidden is then only
 * finite where the weight itself is.
 * The first call on a device looks up the driver's tensor-map encoder (TPPO_ERR_CUDA if absent).
 */
int tppo_lmhead_logprob_fwd_bwd(const void *hidden, const void *weight,
                                int64_t M, int32_t K, int32_t V,
                                const int32_t *targets, const int32_t *aux_idx,
                                const float *old_logp, const float *adv, int64_t aux_len,
                                float eps_low, float eps_high, float denom,
                                float *logp, float *token_loss, float *loss, int32_t *stats,
                                void *dhidden, void *dweight, int32_t chunk_tiles,
                                void *workspace, size_t workspace_bytes, void *stream);

/*
 * The same operation with the vocabulary split across devices (the LM-head weight held as column
 * shards, one per rank; the rows, targets and per-token scalars replicated).  Eq. 1 needs, per row,
 * the maximum logit, the sum of exponentials and the target's logit over the WHOLE vocabulary, so
 * the work is two calls with one exchange between them that the caller performs (the library
 * issues no collective):
 *
 *   1. tppo_lmhead_shard_stats on each rank: over the V_shard columns of its shard (vocabulary ids
 *      v_offset .. v_offset + V_shard - 1), per row r
 *          row_max[r] = max_v x[r,v],  row_sumexp[r] = sum_v exp(x[r,v] - row_max[r]),
 *          row_target_logit[r] = x[r, targets[r]] if the target lies in the shard, else 0.
 *      Rows with a target outside [0, V_total) get (0, 0, 0) and raise the status bit.
 *   2. the merge across ranks, m = max_r m_r;  S = sum_r s_r * exp(m_r - m);  xy = sum_r xy_r:
 *      the caller all-reduces (max) a copy of row_max into row_max_all, calls
 *      tppo_lmhead_shard_rescale, which multiplies row_sumexp[r] by exp(row_max[r] - row_max_all[r])
 *      in place (a skipped row keeps 0), and all-reduces (sum) row_sumexp and row_target_logit.
 *   3. tppo_lmhead_shard_fwd_bwd on each rank with the merged vectors: evaluates Eq. 1 (loss, logp,
 *      token_loss and stats come out identical on every rank), then forms the gradient for its
 *      columns only: dweight_shard [K, V_shard] is complete; dhidden_partial [M, K] holds this
 *      shard's term of dX * weight^T and the caller sums it over the ranks.
 *
 * All arrays live on the device.  row_max, row_sumexp, row_target_logit: [M] fp32.
 *   stats of tppo_lmhead_shard_stats: [4] int32, only the status bits (stats[3]) are written.
 *   workspace for either call: tppo_workspace_bytes(TPPO_OP_LMHEAD, M, K, 0, V_shard) bytes.
 * Every other argument, the limits on K and V_shard (multiples of 8) and the errors are those of
 * tppo_lmhead_logprob_fwd_bwd; 0 <= v_offset <= V_total - V_shard or TPPO_ERR_INVALID_ARG.  With one
 * shard (v_offset = 0, V_shard = V_total) the two calls compute exactly what the unsharded call does.
 */
int tppo_lmhead_shard_stats(const void *hidden, const void *weight_shard,
                            int64_t M, int32_t K, int32_t V_shard, int32_t v_offset, int32_t V_total,
                            const int32_t *targets,
                            float *row_max, float *row_sumexp, float *row_target_logit,
                            int32_t *stats, int32_t chunk_tiles,
                            void *workspace, size_t workspace_bytes, void *stream);
int tppo_lmhead_shard_rescale(const float *row_max, const float *row_max_all, float *row_sumexp,
                              int64_t M, void *stream);
int tppo_lmhead_shard_fwd_bwd(const void *hidden, const void *weight_shard,
                              int64_t M, int32_t K, int32_t V_shard, int32_t v_offset, int32_t V_total,
                              const int32_t *targets, const int32_t *aux_idx,
                              const float *old_logp, const float *adv, int64_t aux_len,
                              float eps_low, float eps_high, float denom,
                              const float *row_max, const float *row_sumexp,
                              const float *row_target_logit,
                              float *logp, float *token_loss, float *loss, int32_t *stats,
                              void *dhidden_partial, void *dweight_shard, int32_t chunk_tiles,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * Successive batching between two training steps (Section 3.2 and its batching figure; the step of
 * Algorithm 1 that keeps the unfinished samples of the last step and puts new prompts in the place
 * of the finished ones).  The batch keeps its B slots, visited in ascending order:
 *   - truncated[i] != 0 (no end condition reached): the sequence stays in slot i; the tokens of this
 *     window join those of earlier windows: next_prompt_len = prompt_len, next_prev_len = prev_len +
 *     new_len, slot_source = -1.
 *   - otherwise the slot is freed and listed in free_slots; the k-th freed slot takes queued prompt
 *     k while the queue lasts (k < M): next_prompt_len = its length, next_prev_len = 0, slot_source =
 *     k; later freed slots stay empty (lengths 0, slot_source = -2).
 * The context of the next step (everything known before generation) is packed slot by slot into
 * next_tokens with offsets next_seq_begin: a kept slot's prompt and all its generated tokens copied
 * from `tokens`, a refilled slot's prompt copied from `queue_tokens`.
 *
 *   seq_begin [B+1], prompt_len / prev_len / new_len [B] int32, truncated [B] u8: the finished step
 *   tokens       [N] int32 token ids in that packed layout
 *   queue_begin  [M+1] int32 offsets of the queued prompts inside queue_tokens [queue_total]
 *   next_prompt_len, next_prev_len [B]; next_seq_begin [B+1]; next_tokens [capacity] int32 out
 *   free_slots   [B] int32 out, ascending, first counts[0] entries valid
 *   slot_source  [B] int32 out
 *   counts       [4] int32 out: freed slots, refilled slots, context tokens of the next step, device
 *                status bits (TPPO_DEV_OVERFLOW when the context exceeds `capacity` or 2^31-1: the
 *                excess is not written; TPPO_DEV_BAD_INDEX for negative lengths and for a slot whose
 *                source range does not lie inside `tokens` / `queue_tokens`: its context is then
 *                written as zeros, nothing outside the arrays is read)
 * No workspace and no clear beforehand: the slot walk writes all four counts itself, and the copy
 * kernel is launched as its programmatic dependent (scheduled while the walk still runs, reading its
 * results only after it has finished).  Bit-exact and run-to-run identical.
 */
int tppo_advance_batch(const int32_t *seq_begin, const int32_t *prompt_len,
                       const int32_t *prev_len, const int32_t *new_len,
                       const uint8_t *truncated, const int32_t *tokens, int64_t N,
                       const int32_t *queue_begin, const int32_t *queue_tokens,
                       int64_t queue_total, int32_t B, int32_t M,
                       int32_t *next_prompt_len, int32_t *next_prev_len,
                       int32_t *next_seq_begin, int32_t *next_tokens, int64_t capacity,
                       int32_t *free_slots, int32_t *slot_source, int32_t *counts,
                       void *stream);

/*
 * ---- Dense operators around the LM-head -----------------------------------------------------------
 * The final layer norm that produces `hidden` and takes `dhidden`, the projections (in 16 and 8 bits) and the
 * value head, the join of a block with the residual stream, the norm of all gradients, and the update they are
 * turned into.  They follow the conventions above
 * with two differences:
 *   - matrices may be strided: element (r, c) is at r * ld + c, ld >= number of columns.  16-byte
 *     aligned rows (base and ld) take the fast paths; any other base (aligned to its element) and ld
 *     is handled.
 *   - `status` ([1] int32, may be NULL) is ADDED TO: bits are set, never cleared, so one word that the
 *     caller zeroes can collect the calls of a whole step.
 * Reductions are done in a fixed order: results are run-to-run identical.  Row and column counts up to
 * 2^30 (TPPO_ERR_UNSUPPORTED beyond).
 */

/*
 * Layer norm of M rows of N elements, statistics in fp32:
 *     mean = sum_c x / N,  rstd = 1 / sqrt(sum_c (x - mean)^2 / N + eps),
 *     y = (x - mean) * rstd * gamma + beta
 *   x [M, N] of `dtype` (TPPO_BF16 or TPPO_F32), y [M, N] of the same type; y may be x itself with
 *   the same row stride
 *   gamma, beta  [N] of `param_dtype` (either type), each may be NULL (1 and 0)
 *   mean, rstd   [M] fp32 out, each may be NULL: what tppo_layer_norm_bwd takes
 *   eps >= 0
 * A row that holds a NaN or an infinity, or whose sum or variance leaves the range of fp32 (with eps = 0 that
 * includes a variance of 0), has no statistics: its y, mean and rstd are written 0 and
 * TPPO_DEV_NONFINITE is raised.  gamma and beta are taken as they are: one that is not finite, or carries a
 * y past the range of its type, leaves such elements in y.
 */
int tppo_layer_norm_fwd(const void *x, int32_t dtype, int64_t M, int32_t N, int64_t ldx,
                        const void *gamma, const void *beta, int32_t param_dtype, float eps,
                        void *y, int64_t ldy, float *mean, float *rstd, int32_t *status,
                        void *stream);

/*
 * Its backward pass.  With h = (x - mean) * rstd and a = dy * gamma:
 *     dx = rstd * (a - sum_c a / N - h * sum_c (a h) / N),
 *     dgamma[c] = sum_r dy * h,   dbeta[c] = sum_r dy
 *   dy, x [M, N] of `dtype`; mean, rstd [M] fp32 from the forward call
 *   dx [M, N] of `dtype` or NULL; may be dy itself with the same row stride (not x)
 *   dgamma, dbeta [N] of `param_dtype`, each may be NULL; overwritten, not accumulated
 *   workspace  tppo_workspace_bytes(TPPO_OP_LAYER_NORM, M, 0, 0, N) bytes; may be NULL when both
 *              dgamma and dbeta are
 * A row without statistics (rstd = 0) contributes nothing and gets dx = 0; so does a row whose dy or x
 * is not finite or whose sums of a and a h are not (a gamma that is not finite makes them so in every row), which
 * raises TPPO_DEV_NONFINITE.  Elements of dx and sums over rows that leave the range
 * of their type become infinities.  M = 0 writes dgamma = dbeta = 0.
 */
int tppo_layer_norm_bwd(const void *dy, const void *x, int32_t dtype, int64_t M, int32_t N,
                        int64_t lddy, int64_t ldx, const void *gamma, int32_t param_dtype,
                        const float *mean, const float *rstd, void *dx, int64_t lddx,
                        void *dgamma, void *dbeta, int32_t *status,
                        void *workspace, size_t workspace_bytes, void *stream);

/* activations of the linear operator */
enum {
    TPPO_ACT_NONE = 0,
    TPPO_ACT_RELU = 1,
    TPPO_ACT_GELU = 2,      /* z * Phi(z)                                                       */
    TPPO_ACT_GELU_TANH = 3, /* z / 2 * (1 + tanh(sqrt(2/pi) * (z + 0.044715 z^3)))              */
    TPPO_ACT_SILU = 4       /* z / (1 + exp(-z))                                                */
};

/*
 * Matrix product with bias, activation and residual in its epilogue:
 *     z = x * weight + bias,   y = act(z) + residual
 *   x [M, K] bf16, weight [K, N] bf16 (the layout of the LM-head weight); any K, N >= 1
 *   bias      [N] of `bias_dtype` or NULL
 *   residual  [M, N] bf16 or NULL; may be y itself when y is bf16 with the same row stride
 *   y         [M, N] of `y_dtype` (fp32 e.g. for a value head, whose N is 1)
 *   preact    [M, N] bf16 out or NULL: z, which tppo_linear_bwd needs unless the activation is
 *             TPPO_ACT_NONE
 *   workspace tppo_workspace_bytes(TPPO_OP_LINEAR, M, K, n_max, N) bytes.  The forward call uses it
 *             only to copy an operand whose rows are not 16-byte aligned -- or, where that makes a large
 *             product faster and there is room, not whole 128-byte lines -- and may be given NULL when x
 *             and weight are 16-byte aligned.  The query counts those copies when K or N is not a
 *             multiple of 64 -- for N <= 4, when K is not a multiple of 8 -- or when n_max is 1: pass that for
 *             misaligned views (base or ld) of matrices of other sizes.  (With N <= 4 such views need no more
 *             than the plain query says; the backward call is faster with the copies from 2^23 elements on.)
 * Products are bf16, sums and the epilogue fp32, y is rounded once.  An element whose z or y is not
 * finite or leaves the range of the type it is stored in is written 0 and raises TPPO_DEV_NONFINITE.
 * No output may overlap x, weight or another output.
 * The first call on a device looks up the driver's tensor-map encoder (TPPO_ERR_CUDA if absent).
 */
int tppo_linear_fwd(const void *x, int64_t ldx, const void *weight, int64_t ldw,
                    int64_t M, int32_t K, int32_t N, const void *bias, int32_t bias_dtype,
                    int32_t activation, const void *residual, int64_t ldr,
                    void *y, int32_t y_dtype, int64_t ldy, void *preact, int64_t ldp,
                    int32_t *status, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Its backward pass.  With dz = dy * act'(z):
 *     dx = dz * weight^T,   dweight = x^T * dz,   dbias[n] = sum_m dz        (dresidual = dy)
 *   dy [M, N] of `dy_dtype`; preact [M, N] bf16 from the forward call (not read, and may be NULL, for
 *   TPPO_ACT_NONE); act' of TPPO_ACT_RELU at 0 is 0
 *   dx [M, K] bf16, dweight [K, N] bf16, dbias [N] of `bias_dtype`: each may be NULL; overwritten, not
 *   accumulated.  No output may overlap an input or another output.
 *   x may be NULL without dweight, weight without dx
 *   workspace as for tppo_linear_fwd: for dz, the partial sums of dbias and operand copies; may be
 *   NULL when none is needed (TPPO_ACT_NONE, aligned bf16 operands, no dbias)
 * dz is rounded to bf16 before the two products where these run on the tensor cores -- always for N > 4, and for
 * fewer columns of more than 2^23 elements of x where rows of x or dx are not 16-byte aligned -- and kept in fp32
 * elsewhere (dbias sums the unrounded values).  An element of dz or of an output that is not finite or leaves the
 * range of bf16 counts or is written as 0 and raises TPPO_DEV_NONFINITE.  One exception: with TPPO_ACT_NONE a bf16
 * dy is the products' operand as it is, so its elements that are not finite make every element of dx and dweight
 * that they enter 0 (dbias leaves them out).  M = 0 writes dweight = dbias = 0.
 */
int tppo_linear_bwd(const void *dy, int32_t dy_dtype, int64_t lddy, const void *x, int64_t ldx,
                    const void *weight, int64_t ldw, int64_t M, int32_t K, int32_t N,
                    int32_t activation, const void *preact, int64_t ldp,
                    void *dx, int64_t lddx, void *dweight, int64_t lddw,
                    void *dbias, int32_t bias_dtype, int32_t *status,
                    void *workspace, size_t workspace_bytes, void *stream);

/*
 * Orthogonalised update of a weight matrix (what its gradient, e.g. dweight of the calls above, is
 * turned into), by Newton-Schulz products:
 *     momentum = mu * momentum + grad,   U = nesterov ? grad + mu * momentum : momentum
 *     X = U / (|U|_F + eps);  `steps` times:  A = X X^T,  B = b A + c A^2,  X = a X + B X
 *     update = scale * X,                (a, b, c) = (3.4445, -4.7750, 2.0315)
 * which multiplies small singular values of X by up to 3.44 per step, keeps those that have come near 1 between
 * 0.68 and 1.21, and leaves the singular vectors.  Five steps bring up what is above some 1.5e-3 of the norm.
 * (The products are taken from the smaller side; the result is the same.)
 *   grad      [R, C] of `grad_dtype`; not changed, unless `update` is grad itself
 *   momentum  [R, C] fp32 in/out, or NULL: U = grad (mu and nesterov are then not used)
 *   eps >= 0; 1 <= steps <= 16 (five is customary)
 *   scale     e.g. sqrt(max(1, R / C)), at most 1e38 in magnitude; the caller applies weight -= lr * update
 *   update    [R, C] bf16 out; may be grad itself when that is bf16 with the same row stride
 *   workspace tppo_workspace_bytes(TPPO_OP_MUON, R, 0, 0, C) bytes
 * Precision: momentum and X are fp32; operands of the products are rounded to fp16, sums are fp32.  The
 * error of X before its rounding to bf16 is about 1e-3 of its norm after five steps.
 * A gradient or momentum element that is not finite, or becomes so, counts as 0 (momentum is written 0
 * there) and raises TPPO_DEV_NONFINITE.  U = 0 gives update = 0.
 */
int tppo_muon_orthogonalize(const void *grad, int32_t grad_dtype, int64_t ldg,
                            float *momentum, int64_t ldm, int64_t R, int32_t C,
                            float mu, int32_t nesterov, float eps, int32_t steps, float scale,
                            void *update, int64_t ldu, int32_t *status,
                            void *workspace, size_t workspace_bytes, void *stream);

/* the norms of the residual join: bits */
enum {
    TPPO_NORM_POST = 1, /* of the block's output, before it joins the residual stream */
    TPPO_NORM_PRE = 2   /* of the joined stream, for the next block                   */
};

/*
 * Residual join: a block's output z is normed, gated and added to the scaled residual stream, and the sum is
 * normed for the next block.  Per row, with root-mean-square norms in fp32:
 *     rstd_post = 1 / sqrt(sum_c z^2 / N + eps),   p = z * rstd_post * gamma_post    (p = z without TPPO_NORM_POST)
 *     h = alpha * residual + gate * p
 *     rstd_pre = 1 / sqrt(sum_c h^2 / N + eps),    n = h * rstd_pre * gamma_pre      (no n without TPPO_NORM_PRE)
 *   z, residual [M, N] of `dtype` (TPPO_BF16 or TPPO_F32)
 *   gate        NULL (1); one row [N] of `param_dtype`, shared by all rows, with ldg = 0; or [M, N] of `dtype`
 *               with ldg >= N
 *   gamma_post, gamma_pre [N] of `param_dtype` or NULL (1; always NULL without their norm)
 *   norms       any combination of the bits above
 *   h           [M, N] of `dtype` out; may be residual itself or z itself with the same row stride
 *   n           [M, N] of `dtype` out, given exactly with TPPO_NORM_PRE; may be z itself (then h may not)
 *   rstd_post, rstd_pre [M] fp32 out or NULL: what the backward call takes
 *   alpha finite, eps >= 0
 * Each output is rounded once; n is formed from the unrounded h.  A row that has no statistics (a NaN or
 * infinity in it, in its gate or in gamma_post; sums of squares or of magnitudes beyond fp32; a mean square plus eps
 * below 2^-126, which with eps = 0 is a row of zeros or of numbers whose squares lose bits in fp32) gets h, n and
 * rstd of 0 and raises TPPO_DEV_NONFINITE.  gamma_pre is taken as it is,
 * and elements that leave the range of their type become infinities.
 */
int tppo_residual_norm_fwd(const void *z, int64_t ldz, const void *residual, int64_t ldr,
                           const void *gate, int64_t ldg, int32_t dtype, int64_t M, int32_t N,
                           const void *gamma_post, const void *gamma_pre, int32_t param_dtype,
                           float alpha, float eps, int32_t norms, void *h, int64_t ldh, void *n, int64_t ldn,
                           float *rstd_post, float *rstd_pre, int32_t *status, void *stream);

/*
 * Its backward pass.  With hh = h * rstd_pre, zz = z * rstd_post (z without TPPO_NORM_POST):
 *     d = dh + rstd_pre * (dn * gamma_pre - hh * sum_c (dn * gamma_pre * hh) / N)     (d = dh without TPPO_NORM_PRE)
 *     dresidual = alpha * d,   dgate = d * zz * gamma_post,   a = d * gate * gamma_post,
 *     dz = rstd_post * (a - zz * sum_c (a * zz) / N)                                  (dz = a without TPPO_NORM_POST)
 *     dgamma_post[c] = sum_r d * gate * zz,   dgamma_pre[c] = sum_r dn * hh,   and dgate summed over r for a row
 *   dh          [M, N] of `dtype` or NULL (0): gradient of h from further down the residual stream
 *   dn          [M, N] of `dtype`, given exactly with TPPO_NORM_PRE
 *   z; h as the forward call stored it (with TPPO_NORM_PRE only, else NULL); rstd_post, rstd_pre of its norms
 *   dz, dresidual [M, N] of `dtype`, each may be NULL; dresidual may be dh itself, dz may be dn itself, with the same
 *               row stride
 *   dgate       like gate ([N] of `param_dtype` with ldg = 0, or [M, N] of `dtype` with row stride lddg) or NULL
 *   dgamma_post, dgamma_pre [N] of `param_dtype` or NULL; overwritten, not accumulated
 *   workspace   tppo_workspace_bytes(TPPO_OP_RESIDUAL_NORM, M, 0, 0, N) bytes
 * A row without statistics (an rstd of 0) contributes nothing and gets gradients of 0; so does a row in which a
 * gradient, activation or parameter that enters a product above is not finite or makes its sums so, which raises
 * TPPO_DEV_NONFINITE.  Elements and sums over rows that leave the range of their type become infinities.  M = 0
 * writes the column sums 0.
 */
int tppo_residual_norm_bwd(const void *dh, int64_t lddh, const void *dn, int64_t lddn, const void *z, int64_t ldz,
                           const void *h, int64_t ldh, const void *gate, int64_t ldg, int32_t dtype,
                           int64_t M, int32_t N, const void *gamma_post, const void *gamma_pre, int32_t param_dtype,
                           const float *rstd_post, const float *rstd_pre, float alpha, int32_t norms,
                           void *dz, int64_t lddz, void *dresidual, int64_t lddr, void *dgate, int64_t lddg,
                           void *dgamma_post, void *dgamma_pre, int32_t *status,
                           void *workspace, size_t workspace_bytes, void *stream);

/* how elements share a scale: bits of the quantiser's and the product's `block` */
enum {
    TPPO_FP8_ROWS = 1,  /* 128 consecutive elements along the contraction                      */
    TPPO_FP8_SQUARE = 2 /* 128 x 128 elements (weights: one scale serves both of their layouts) */
};

/*
 * 8-bit values (e4m3: four significant bits, up to 448) with one fp32 scale per block of 128: x ~ q * scale.  The
 * scale is the least power of two 2^e, e >= -126, for which the block's largest magnitude is at most 448 * 2^e (1 for
 * a block of zeros), so that q is x / scale rounded once (to nearest even), and q * scale is exact in fp32 -- in bf16 too
 * from a scale of 2^-124 on, below which bf16's smallest numbers are coarser.  q holds the rows of x as they are, for products that contract over x's columns; qt is x
 * transposed, for products that contract over x's rows, with blocks of its own along them.
 *   x       [M, K] of `dtype` (TPPO_BF16 or TPPO_F32)
 *   q       [M, K] 8-bit out or NULL;  scale out:
 *             TPPO_FP8_ROWS    [ceil(K / 128), M] with row stride lds: scale of (row m, columns 128 b ..) at (b, m)
 *             TPPO_FP8_SQUARE  [ceil(M / 128), ceil(K / 128)] with row stride lds
 *   qt      [K, M] 8-bit out or NULL;  scale_t out:
 *             TPPO_FP8_ROWS    [ceil(M / 128), K] with row stride ldst
 *             TPPO_FP8_SQUARE  [ceil(K / 128), ceil(M / 128)] with row stride ldst: the transpose of scale
 * q, qt: base and row stride multiples of 16 bytes (one row needs no stride).  Padding between rows is not written.  An element that is not finite counts as 0 and raises TPPO_DEV_NONFINITE.
 */
int tppo_fp8_quantize(const void *x, int32_t dtype, int64_t ldx, int64_t M, int64_t K, int32_t block,
                      void *q, int64_t ldq, float *scale, int64_t lds,
                      void *qt, int64_t ldqt, float *scale_t, int64_t ldst, int32_t *status, void *stream);

/*
 * Product of two such matrices, both given with the contraction along their rows:
 *     y[m, n] = sum_b a_scale(b, m) * b_scale(b, n) * sum_{k in block b} a[m, k] * b[n, k]
 *   a        [M, K], a_scale [ceil(K / 128), M] as TPPO_FP8_ROWS gives them
 *   b        [N, K], b_scale as `b_block` says: TPPO_FP8_ROWS [ceil(K / 128), N], or TPPO_FP8_SQUARE
 *            [ceil(N / 128), ceil(K / 128)]
 *   y        [M, N] of `y_dtype`, rounded once
 * With a weight w [K, N] quantised in squares (q, qt), activations x and gradients dy in rows (q, qt):
 *     x w        = product of x's q  and w's qt (TPPO_FP8_SQUARE)
 *     dy w^T     = product of dy's q and w's q  (TPPO_FP8_SQUARE)
 *     x^T dy     = product of x's qt and dy's qt (TPPO_FP8_ROWS)
 * Scales are powers of two, 2^-126 to 2^127; products and sums are those of the tensor cores, in fp32.  An element of y
 * that is not finite, leaves the range of its type or has a scale of another kind in it is written 0 and raises
 * TPPO_DEV_NONFINITE.  K = 0 gives y = 0.  Alignment of a and b as for the quantiser; y may be strided at any element.  y may not overlap an input.
 * The first call on a device looks up the driver's tensor-map encoder (TPPO_ERR_CUDA if absent).
 */
int tppo_fp8_matmul(const void *a, int64_t lda, const float *a_scale, int64_t ldas,
                    const void *b, int64_t ldb, const float *b_scale, int64_t ldbs, int32_t b_block,
                    int64_t M, int64_t N, int64_t K, void *y, int32_t y_dtype, int64_t ldy,
                    int32_t *status, void *stream);

/* For tests, host only: how tppo_fp8_matmul cuts a product -- 16 times the rows of y that a tile of its split kernel takes
 * (0: the persistent kernel), plus the blocks that share a tile's contraction.  aligned_rows: y's rows start on 16-byte
 * boundaries.  -1 for sizes outside [1, 2^30]. */
int32_t tppo_test_fp8_cut(int64_t M, int64_t N, int64_t K, int32_t y_dtype, int32_t aligned_rows);

/* One of many tensors: n contiguous elements of `dtype` (TPPO_BF16 or TPPO_F32) at the device address `data`,
 * which may be NULL when n is 0.  Any alignment of its element. */
typedef struct {
    void *data;
    int64_t n;
    int32_t dtype;
    int32_t reserved; /* 0 */
} tppo_tensor;

/*
 * Sum of squares and norm over all elements of `count` gradients:
 *     sum_sq = sum_i sum_e g_i[e]^2   (64 bits),   norm = sqrt(sum_sq)   (fp32)
 *   grads     HOST array of `count` tensors, read before the call returns; the addresses become part of the
 *             launch (a captured call keeps them).  A tensor listed twice counts twice.
 *   sum_sq    [1] fp64 out;  norm [1] fp32 out or NULL
 *   workspace tppo_workspace_bytes(TPPO_OP_GRAD_NORM, count, 0, 0, 0) bytes
 * With a gradient element that is not finite both results are +infinity and TPPO_DEV_NONFINITE is raised; a norm
 * beyond fp32 is +infinity as well, sum_sq is then still right.  With several ranks, each holding some of the gradients, add up their sum_sq and
 * pass the sum to tppo_grad_clip.
 */
int tppo_grad_norm(const tppo_tensor *grads, int32_t count, double *sum_sq, float *norm, int32_t *status,
                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * Gradients scaled down to a norm of at most max_norm:
 *     coef = min(1, max_norm / sqrt(sum_sq)),   out_i = coef * g_i
 *   sum_sq    [1] fp64 from tppo_grad_norm, on the device;  max_norm finite, >= 0
 *   out       HOST array of `count` tensors of the same lengths, of either type each; or NULL: in place.  An
 *             output is its gradient itself, of the same type, or overlaps no gradient and no other output.  A gradient
 *             that is listed twice and in place both times is scaled once.  In place, a coefficient of 1 leaves the
 *             gradients untouched (and unread).
 *   coef      [1] fp32 out or NULL
 * A sum_sq that is not finite gives coef = 0, outputs of 0 and TPPO_DEV_NONFINITE: a step without effect.
 */
int tppo_grad_clip(const tppo_tensor *grads, int32_t count, const double *sum_sq, double max_norm,
                   const tppo_tensor *out, float *coef, int32_t *status, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TPPO_H */
