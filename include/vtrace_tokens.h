/*
 * libvtrace, the learner step of a policy over a token vocabulary: what
 * vtrace.h computes for a handful of actions, for action sets (vocabularies) so
 * large that the logits [T,B,V] are never formed.  One training step is
 *
 *   vtrace_vocab_log_probs     hidden states, vocabulary layer -> log pi(a_t|x_t),
 *                              entropy and log-sum of every step
 *   vtrace_log_prob_loss_grad  log-probabilities -> V-trace losses and their
 *                              gradients with respect to log pi(a_t|x_t), the
 *                              entropies and the values
 *   vtrace_vocab_grad          those gradients -> gradients of the hidden states and
 *                              of the vocabulary layer
 *   vtrace_clip_grad_norm      the global norm of all gradients, and clipping by it
 *
 * Cross entropy is the same with d_log_probs = -1 (or -1/steps) and no entropy.
 *
 * Conventions (device pointers, status codes, streams, no allocation, no
 * synchronisation) and layouts are those of vtrace.h.  Outputs must not alias
 * inputs or each other, except where stated.  Calls are re-entrant; concurrent
 * calls need distinct workspaces, and calls in turn, of whatever kind, may share
 * one (vtrace_workspace_bytes).  Repeated calls on the same inputs give
 * bit-identical results.  Every call may be captured into a HIP graph.
 */
#ifndef VTRACE_TOKENS_H_
#define VTRACE_TOKENS_H_

#include "vtrace.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The token of a step that takes no part: a prompt, or the padding behind a
 * sequence.  Its hidden state is not used (it may hold NaN), its outputs are 0
 * and it adds nothing to any gradient.
 */
#define VTRACE_NO_TOKEN (-1)

/*
 * Log-probabilities of a vocabulary layer, without keeping its logits.  With
 *   z[t,b,v] = <hidden[t,b,:], vocab_weight[v,:]> + vocab_bias[v],
 *   L = log sum_v exp z[t,b,v]:
 *
 *   log_probs  [T,B] float32: log pi(a_t|x_t) = z[t,b,a_t] - L
 *   log_sums   [T,B] float32: L (vtrace_vocab_grad takes it)
 *   entropy    optional [T,B] float32: -sum_v pi log pi (a token with pi = 0 adds 0)
 *
 *   T, B           T*B <= 2^25
 *   V              1 .. 2^24 tokens, T*B*V <= 2^38
 *   H              hidden size, a multiple of 8 from 8 to 32768; T*B*H < 2^30
 *   hidden         [T,B,H] bfloat16, 16-byte aligned
 *   vocab_weight   [V,H] bfloat16, 16-byte aligned: a row for each token
 *   vocab_bias     optional [V] float32 (NULL = 0); -INFINITY, or anything below -1e37,
 *                  rules a token out
 *   tokens         [T,B] int32: 0 <= a < V, or VTRACE_NO_TOKEN
 *   workspace      vtrace_vocab_workspace_bytes(T,B,V,H) bytes, 16-byte aligned,
 *                  cleared once by vtrace_workspace_init
 * Numerics: bfloat16 products accumulated in float32 from the bias, exponentials
 * in float32 of differences to the largest logit of a piece, their sums in float32
 * over the piece and joined in float64.  A piece is the 64 or 128 tokens of one
 * wave, or, up to 128 steps, the tokens of one workgroup: V / 1024 to V / 256, at
 * least 16.  Any other token makes that step's log_probs NaN and raises the
 * workspace's flag (vtrace_error_flag).  A step whose tokens are all ruled out has
 * log_sums -INFINITY and NaN elsewhere; a finite bias of -1e9 or less has the same
 * effect beside allowed tokens.  NaN and Inf inputs are propagated, also from the
 * row of a token that is ruled out (0 * NaN): such rows have to hold numbers.
 */
size_t vtrace_vocab_workspace_bytes(int64_t T, int64_t B, int64_t V, int64_t H);

vtrace_status vtrace_vocab_log_probs(
    int64_t T, int64_t B, int64_t V, int64_t H,
    const void* hidden, const void* vocab_weight, const float* vocab_bias, const int32_t* tokens,
    float* log_probs, float* log_sums, float* entropy,
    void* workspace, size_t workspace_bytes, vtrace_stream_t stream);

/*
 * The gradients of a loss through log_probs and entropy, with the logits formed
 * again in pieces of the vocabulary.  With
 *   G[t,b,v] = d_log_probs[t,b] (1[v = a_t] - pi_v) - d_entropy[t,b] pi_v (log pi_v + entropy[t,b]):
 *
 *   d_hidden   [T,B,H] = sum_v G[t,b,v] vocab_weight[v,:], grad_dtype
 *   d_weight   [V,H] = sum over (t,b) of G[t,b,v] hidden[t,b,:], grad_dtype
 *   d_bias     [V] float32 = sum over (t,b) of G[t,b,v]; NULL to skip
 *
 *   log_sums, entropy   what vtrace_vocab_log_probs returned for these inputs
 *   d_log_probs         [T,B] float32; d_entropy [T,B] float32, or NULL for none
 *                       (entropy is then not read and may be NULL)
 *   grad_dtype          VTRACE_F32 or VTRACE_BF16; d_hidden, d_weight 16-byte aligned
 *   workspace           vtrace_vocab_grad_workspace_bytes(T,B,V,H,grad_dtype) bytes
 * Everything else as above.  grad_dtype is also the choice of how G enters its two
 * products: as one bfloat16 (2^-8 a term) for bfloat16 outputs, and as a bfloat16
 * pair (high + low part, 2^-17 a term) for float32 ones; sums over steps and tokens
 * are float32 (d_bias: 64 or 128 steps, then float64).  With few steps nothing
 * averages G's rounding out, and a bfloat16 output has two.  pi_v is
 * exp(z - log_sums): the float32 rounding of a log-sum of magnitude M, M 2^-24,
 * is pi's relative error.  A G below 2^-126 may count as 0.  A token that is
 * neither in the vocabulary nor VTRACE_NO_TOKEN makes that step's G NaN, and with
 * it d_weight and d_bias.
 */
size_t vtrace_vocab_grad_workspace_bytes(int64_t T, int64_t B, int64_t V, int64_t H,
                                         vtrace_dtype grad_dtype);

vtrace_status vtrace_vocab_grad(
    int64_t T, int64_t B, int64_t V, int64_t H, vtrace_dtype grad_dtype,
    const void* hidden, const void* vocab_weight, const float* vocab_bias, const int32_t* tokens,
    const float* log_sums, const float* entropy, const float* d_log_probs, const float* d_entropy,
    void* d_hidden, void* d_weight, float* d_bias,
    void* workspace, size_t workspace_bytes, vtrace_stream_t stream);

/*
 * The losses and gradients of vtrace_loss_grad from log-probabilities instead of
 * logits, for lanes (answers) of different lengths.
 *
 *   target_log_probs     [T,B] float32 log pi(a_t|x_t)
 *   behaviour_log_probs  [T,B] float32 log mu(a_t|x_t)
 *   entropy              optional [T,B] float32: the policy's entropy; NULL leaves the
 *                        entropy loss 0
 *   rewards, discounts, values [T,B], bootstrap_value [B]   as in vtrace.h
 *   lengths              optional [B] int32 (device): lane b has steps 0 .. lengths[b] - 1, its
 *                        bootstrap value follows the last of them; values outside
 *                        [0, T] count as 0 or T.  NULL: every lane has T steps.  Inputs
 *                        behind a lane's last step are not used; outputs there are 0.
 *   variant              as in vtrace_loss_grad_ex (NULL = V-trace); behaviour_input
 *                        and grad_dtype are not used but have to be valid
 *   losses       [4] float32 {total, policy gradient, baseline, entropy}
 *   d_log_probs  [T,B] float32: -pg_adv (times pi / (pi + epsilon) for epsilon-correction)
 *   d_entropy    [T,B] float32: -entropy_cost on a lane's steps; NULL to skip.  The
 *                entropy loss is -entropy_cost * sum of entropy, as in vtrace.h
 *   d_values     [T,B] float32: baseline_cost (V(x_t) - v_t)
 *   vs, pg_advantages  optional [T,B] float32
 *   workspace    vtrace_log_prob_workspace_bytes(T,B) bytes, 16-byte aligned, cleared
 *                once by vtrace_workspace_init
 * T*B <= 2^40, B <= 2^22.  Ratios, recursion and loss sums are float64.
 */
size_t vtrace_log_prob_workspace_bytes(int64_t T, int64_t B);

vtrace_status vtrace_log_prob_loss_grad(
    int64_t T, int64_t B, const float* target_log_probs, const float* behaviour_log_probs,
    const float* entropy, const float* rewards, const float* discounts, const float* values,
    const float* bootstrap_value, const int32_t* lengths, float rho_bar, float c_bar, float lambda,
    float baseline_cost, float entropy_cost, const vtrace_variant* variant,
    float* losses, float* d_log_probs, float* d_entropy, float* d_values,
    float* vs, float* pg_advantages,
    void* workspace, size_t workspace_bytes, vtrace_stream_t stream);

/*
 * Clipping by the global norm (the paper's learner clips its gradients so, App. D):
 *   norm = sqrt(sum over all gradients of g^2),
 *   outputs[i] = gradients[i] * max_norm / max(norm, max_norm).
 *
 *   count       0 .. 2^16 gradients; gradients, outputs, sizes and dtypes are HOST
 *               arrays of that length, read during the call
 *   gradients   device pointers to sizes[i] (0 .. 2^36) contiguous elements of dtypes[i]
 *               (VTRACE_F32 or VTRACE_BF16), element-aligned (NULL if sizes[i] is 0)
 *   outputs     where the clipped gradients go, of the same sizes and types.  An output may be
 *               its own gradient (clipping in place); it may not overlap anything
 *               else of the call: VTRACE_ERR_PARAM, also for the same gradient
 *               twice where it is clipped in place.  NULL: the norm alone.  Copies take a
 *               third of the time where an output lies in 16 bytes as its gradient does
 *   max_norm    >= 0, +INFINITY allowed (no clipping); not used without outputs
 *   norm        [1] float32 device
 *   workspace   VTRACE_CLIP_WORKSPACE_BYTES, 16-byte aligned, cleared once by
 *               vtrace_workspace_init
 * Squares and their sum are float64 (neither overflows nor underflows), the
 * factor is float32.  NaN or Inf gradients are propagated by these formulas:
 * a NaN anywhere makes the norm and every output NaN, an infinite norm gives 0
 * for finite elements and NaN for infinite ones.
 */
#define VTRACE_CLIP_WORKSPACE_BYTES 20736

vtrace_status vtrace_clip_grad_norm(
    int64_t count, const void* const* gradients, void* const* outputs, const int64_t* sizes,
    const int32_t* dtypes, float max_norm, float* norm,
    void* workspace, size_t workspace_bytes, vtrace_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* VTRACE_TOKENS_H_ */
