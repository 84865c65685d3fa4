/*
 * libvtrace, the learner step of a policy over a token vocabulary: what the calls of
 * vtrace_tokens.h leave to do at the network's other end and with its gradients.
 *
 *   vtrace_vocab_embed       tokens -> the network's inputs, rows of the vocabulary's
 *                            table
 *   vtrace_vocab_embed_grad  the inputs' gradients -> the table's, alone or on top of
 *                            what vtrace_vocab_grad left (a layer that shares its rows
 *                            with the inputs)
 *   vtrace_orthogonalize     updates of the network's matrices (clipped gradients, or
 *                            averages of them) -> nearly orthogonal ones
 *
 * Conventions (device pointers, status codes, streams, no allocation, no
 * synchronisation) and layouts are those of vtrace.h.  Outputs must not alias inputs or
 * each other, except where stated.  Calls are re-entrant; concurrent calls need distinct
 * workspaces, and calls in turn, of whatever kind, may share one.  Repeated calls on the
 * same inputs give bit-identical results.  Every call may be captured into a HIP graph.
 */
#ifndef VTRACE_PARAMETERS_H_
#define VTRACE_PARAMETERS_H_

#include "vtrace_tokens.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * embedded[t,b,:] = scale * vocab_weight[tokens[t,b],:], zeros for VTRACE_NO_TOKEN.
 *
 *   T, B           T*B <= 2^25
 *   V, H           tokens, 1 .. 2^24; a row's size, a multiple of 8 from 8 to 32768;
 *                  V*H and T*B*H <= 2^37
 *   vocab_weight   [V,H] of weight_dtype (VTRACE_F32 or VTRACE_BF16), 16-byte aligned
 *   tokens         [T,B] int32: 0 <= a < V, or VTRACE_NO_TOKEN
 *   scale          finite
 *   embedded       [T,B,H] of embedded_dtype, 16-byte aligned
 *   workspace      NULL, or any workspace (16-byte aligned, cleared once by
 *                  vtrace_workspace_init, at least 256 bytes), whose flag
 *                  (vtrace_error_flag) a token that is neither in the vocabulary nor
 *                  VTRACE_NO_TOKEN raises
 * The product is float32, rounded once.  A token that is neither gives a row of NaN.
 */
vtrace_status vtrace_vocab_embed(
    int64_t T, int64_t B, int64_t V, int64_t H, vtrace_dtype weight_dtype, vtrace_dtype embedded_dtype,
    const void* vocab_weight, const int32_t* tokens, float scale, void* embedded,
    void* workspace, size_t workspace_bytes, vtrace_stream_t stream);

/*
 * d_weight[v,:] = scale * sum over the steps with tokens[t,b] = v of d_embedded[t,b,:]
 *                 (+ d_weight[v,:] as it was, with accumulate).
 *
 *   d_embedded   [T,B,H] of embedded_dtype, 16-byte aligned; rows of steps without a
 *                token are not used
 *   d_weight     [V,H] of grad_dtype, 16-byte aligned.  accumulate 0: all of it is
 *                written, rows of tokens that no step has with zeros; otherwise
 *                rows of tokens that steps have are added to, and no other is touched
 *   workspace    vtrace_vocab_embed_grad_workspace_bytes(T,B,V,H) bytes, 16-byte aligned,
 *                cleared once by vtrace_workspace_init.  No smaller T*B, V and H need more
 * Everything else as above.  Sums are float32 over up to 128 steps of a token and float64
 * beyond, in an order that depends on the tokens alone; scaled and added in float32,
 * rounded once.  A token that is neither in the vocabulary nor VTRACE_NO_TOKEN adds
 * nothing and raises the workspace's flag.
 */
size_t vtrace_vocab_embed_grad_workspace_bytes(int64_t T, int64_t B, int64_t V, int64_t H);

vtrace_status vtrace_vocab_embed_grad(
    int64_t T, int64_t B, int64_t V, int64_t H, vtrace_dtype embedded_dtype, vtrace_dtype grad_dtype,
    const void* d_embedded, const int32_t* tokens, float scale, int32_t accumulate, void* d_weight,
    void* workspace, size_t workspace_bytes, vtrace_stream_t stream);

/*
 * Newton-Schulz products that leave a matrix's singular vectors and bring its singular
 * values near 1 (the iteration of Bjorck and Bowie, 1971, with the quintic's coefficients of
 * Jordan et al., "Muon", 2024), for each matrix G of a list on its own:
 *   X = G / max(|G|, epsilon), |G| = sqrt(sum of squares);
 *   `steps` times, with coefficients a, b, c of that step:
 *     A = X X^T,  X <- a X + (b A + c A A) X   (a singular value s becomes a s + b s^3 + c s^5);
 *   output = scale * X.
 *
 *   count         0 .. 2^16 matrices; matrices, outputs, rows, columns, dtypes and scales are
 *                 HOST arrays of that length, coefficients one of 3*steps floats, all
 *                 read during the call
 *   matrices      device pointers to rows[i] x columns[i] (each 0 .. 65536, their product up to 2^31)
 *                 contiguous elements of dtypes[i] (VTRACE_F32 or VTRACE_BF16), element-aligned
 *                 (NULL if there are none)
 *   outputs       where the results go, of the same sizes and types.  An output may be its own
 *                 matrix; it may not overlap anything else of the call: VTRACE_ERR_PARAM
 *   scales        finite factors, NULL = 1
 *   steps         1 .. 64
 *   coefficients  under which singular values from [0, 1] stay within [0, 3.5] in size at every
 *                 step, and eigenvalues of b A + c A A within a range of 12: anything else is
 *                 VTRACE_ERR_PARAM.  Those of the quintic 3.4445, -4.7750, 2.0315 for 5 steps
 *                 bring singular values from 0.01 |G| on into 0.68 .. 1.21
 *   epsilon       finite, > 0; a matrix of zeros gives zeros
 *   workspace     vtrace_orthogonalize_workspace_bytes(count, rows, columns, dtypes) bytes, 16-byte
 *                 aligned, cleared once by vtrace_workspace_init; 0 for an invalid list.  Any list of
 *                 some of the matrices, in any order, needs as many or fewer
 * Numerics: norms are float64.  Matrices of at most 32 rows or columns are float64 up to the
 * result's rounding (as long as the coefficients a multiply to at most 8192 over the steps).
 * Otherwise X has 22 bits (bfloat16 matrices) or is float32 from step to step, sums of
 * products are float32, products take float16 operands of a fixed scale, for float32 matrices
 * in two parts (22 bits) each, and the diagonals of the symmetric matrices are float32.  In
 * relation to their norm, against products in 64 bits and for 5 steps of the quintic, results of
 * bfloat16 matrices are off by little more than their own rounding (1.67e-3 to 1.85e-3, and where
 * one size is some 30 and the other thousands 1.96e-3; the rounding is 1.66e-3), and those of
 * float32 matrices by 3e-7 to 9e-7 (2.4e-6 measured where all but the largest singular values are
 * a hundredth of those).  That holds down to norms of epsilon: far below it, where singular values
 * stay small, results of bfloat16 matrices are off by up to 2^-36 each.  Where terms are all
 * alike (matrices of a few values in large blocks) roundings do not cancel, and results are off by
 * up to 2e-2 (bfloat16); float32 2e-5 where sizes are some hundreds, 3e-4 for thousands and 1.1e-3
 * for 65536 x 32768.  NaN or Inf in a matrix makes all of its result NaN, and that of no other
 * matrix.
 */
size_t vtrace_orthogonalize_workspace_bytes(int64_t count, const int64_t* rows, const int64_t* columns,
                                            const int32_t* dtypes);

vtrace_status vtrace_orthogonalize(
    int64_t count, const void* const* matrices, void* const* outputs, const int64_t* rows,
    const int64_t* columns, const int32_t* dtypes, const float* scales, int32_t steps,
    const float* coefficients, float epsilon,
    void* workspace, size_t workspace_bytes, vtrace_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* VTRACE_PARAMETERS_H_ */
