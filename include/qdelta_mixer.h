/* Entry points of libqdelta.so for the operators that stand around the
 * recurrence in a block: the short causal convolution, the row normalisation
 * and the selective state space scan.  They return the status codes of
 * qdelta.h and follow its conventions (device pointers, validation of every
 * host-visible argument before the first launch, asynchronous on the caller's
 * stream, no device allocation, every output fully overwritten), with three
 * differences: tensors need the alignment of their elements only (16-byte
 * aligned rows run faster), the rows of an input named with a stride
 * (ldx, ldg, ldb, ldc) may lie in a wider tensor, stride elements apart, and
 * an output must not overlap an input unless that is said here.
 *
 * Sequences: cu_seqlens NULL is a dense batch of N sequences of T tokens
 * (token (n, t) is row n T + t); else N sequences are packed into T tokens as
 * in qdelta.h (int32[N + 1] on the device, cu[0] = 0, cu[N] = T).  Where cu[N]
 * < T the tokens from cu[N] on are not read into any result and their rows of
 * the outputs stay as they are.  A malformed cu_seqlens leaves the outputs of
 * the sequences concerned unspecified; memory is never accessed out of bounds.
 *
 * Sizes: a call has less than 2^31 tokens (N T where dense) with T at most
 * 2^31 - 64, and one whose launches would need 2^32 threads or more is
 * QDELTA_EUNSUPPORTED (for the scan about 2^23 heads over all sequences, 2^23
 * groups over all chunks of 64 tokens, or 2^31 heads over all tokens).
 *
 * Precision: sums, statistics and states are fp32.  Exponentials (SiLU, softplus,
 * the state's decays) are good to the last places of fp32, but for decays between
 * two tokens of a chunk, off by |x| 2^-24 relative (their argument is rounded),
 * and, with bf16 activations, for those and SiLU, off by |x| 2^-23. */
#ifndef QDELTA_MIXER_H
#define QDELTA_MIXER_H

#include "qdelta.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- short causal convolution, one filter per channel
 *
 *   u_t = bias + sum_j weight[:, j] x_{t - W + 1 + j};  y = silu ? u sigmoid(u) : u
 *
 *   x [tokens, D] (rows ldx apart), weight [D, W], bias [D] or NULL, y [tokens, D]   (dtype)
 *   initial_state [N, W - 1, D] or NULL (zeros): the W - 1 rows before each
 *   sequence, the oldest first; final_state the same after it, or NULL (dtype)
 * W is 2, 3 or 4 (else QDELTA_EUNSUPPORTED).  Sums are fp32. */
int qdelta_conv_fwd(int32_t N, int32_t T, const int32_t* cu_seqlens, int32_t D, int32_t W, int32_t dtype, int32_t silu,
                    const void* x, int64_t ldx, const void* weight, const void* bias, const void* initial_state,
                    void* y, void* final_state, hipStream_t stream);

/* Its backward.  d_final_state [N, W - 1, D] or NULL (zeros); dx [tokens, D];
 * dweight [D, W], dbias [D] and d_initial_state may be NULL.  The weight's
 * gradients are summed in a fixed order (results do not change from run to
 * run).  Workspace of qdelta_conv_workspace_bytes. */
size_t qdelta_conv_workspace_bytes(int32_t N, int32_t T, int32_t packed, int32_t D, int32_t W);
int qdelta_conv_bwd(int32_t N, int32_t T, const int32_t* cu_seqlens, int32_t D, int32_t W, int32_t dtype, int32_t silu,
                    const void* x, int64_t ldx, const void* weight, const void* bias, const void* initial_state,
                    const void* dy, const void* d_final_state, void* dx, void* dweight, void* dbias,
                    void* d_initial_state, void* ws, size_t ws_bytes, hipStream_t stream);

/* One token of N sequences: x [N, D] (rows ldx apart) and state [N, W - 1, D]
 * into y [N, D] and state_out, which may be state itself. */
int qdelta_conv_step(int32_t N, int32_t D, int32_t W, int32_t dtype, int32_t silu, const void* x, int64_t ldx,
                     const void* weight, const void* bias, const void* state, void* state_out, void* y,
                     hipStream_t stream);

/* ---- row normalisation
 *
 *   xh = (x - mean) rstd,  rstd = 1 / sqrt(var + eps);  rms: mean = 0, var = mean(x^2)
 *   y  = (xh weight + bias) gate sigmoid(gate)
 *
 *   x, gate (or NULL) [rows, D] (rows ldx, ldg apart), weight, bias [D] or NULL, y [rows, D]  (dtype)
 *   stats [rows, 2] float32: mean and rstd, for the backward; or NULL
 * D is at most 8192 (else QDELTA_EUNSUPPORTED).  Statistics are fp32, the
 * variance is taken about the mean. */
int qdelta_norm_fwd(int64_t rows, int32_t D, int32_t dtype, int32_t rms, float eps, const void* x, int64_t ldx,
                    const void* weight, const void* bias, const void* gate, int64_t ldg, void* y, float* stats,
                    hipStream_t stream);

/* Its backward, from the statistics: dx, dgate (with a gate) [rows, D],
 * dweight and dbias [D] (NULL where not wanted), the latter summed over the
 * rows in a fixed order.  Workspace of qdelta_norm_workspace_bytes where
 * either of the two is wanted. */
size_t qdelta_norm_workspace_bytes(int64_t rows, int32_t D);
int qdelta_norm_bwd(int64_t rows, int32_t D, int32_t dtype, int32_t rms, const void* x, int64_t ldx,
                    const void* weight, const void* bias, const void* gate, int64_t ldg, const float* stats,
                    const void* dy, void* dx, void* dweight, void* dbias, void* dgate, void* ws, size_t ws_bytes,
                    hipStream_t stream);

/* ---- selective state space scan with one decay per head
 *
 *   dt  = softplus ? log(1 + exp(raw + dt_bias)) : raw + dt_bias
 *   S_t = exp(dt A) S_{t-1} + dt x_t B_t^T          (S [P, Ns] per sequence and head)
 *   y_t = S_t C_t + D x_t
 *
 *   x [tokens, H, P], B, C [tokens, G, Ns]   (dtype; tokens ldx, ldb, ldc elements apart),
 *                                            head h reads group h / (H / G) of B and C
 *   dt [tokens, H], A [H], D, dt_bias [H] or NULL           float32 (dt A <= 0 expected)
 *   initial_state, final_state [N, H, P, Ns] or NULL        float32 (NULL: zero, not wanted)
 *   y [tokens, H, P]   (dtype)
 * dt A > 0 is taken as well; growth past fp32 (e^88) within 64 tokens leaves
 * infinities or NaN.  P is at most 256, Ns at most 128 and G divides H (else
 * QDELTA_EUNSUPPORTED, QDELTA_EINVAL).  Prompts go by chunks of 64 tokens on the
 * matrix cores: bf16 products of values that are fp32 take them as sums of three
 * bf16 values, which are exact, so that every result keeps fp32's precision until
 * it is rounded to its type.  An infinity in x, B, C or a state may come out as a
 * NaN in what it enters.  Packing does not change a sequence's chunks.  Workspace
 * of qdelta_scan_workspace_bytes. */
size_t qdelta_scan_workspace_bytes(int32_t N, int32_t T, int32_t packed, int32_t H, int32_t G, int32_t P, int32_t Ns,
                                   int32_t is_bwd);
int qdelta_scan_fwd(int32_t N, int32_t T, const int32_t* cu_seqlens, int32_t H, int32_t G, int32_t P, int32_t Ns,
                    int32_t dtype, int32_t softplus, const void* x, int64_t ldx, const float* dt, const float* A,
                    const void* B, int64_t ldb, const void* C, int64_t ldc, const float* D, const float* dt_bias,
                    const float* initial_state, void* y, float* final_state, void* ws, size_t ws_bytes,
                    hipStream_t stream);

/* Its backward, from the inputs alone: dx [tokens, H, P], dB, dC [tokens, G,
 * Ns] (dtype), ddt [tokens, H] (of raw), dA, dD, ddt_bias [H], d_initial_state
 * (float32; the last three may be NULL).  Sums over heads, chunks and tokens
 * run in a fixed order.  A NaN or infinity spoils the gradients of its whole
 * chunk. */
int qdelta_scan_bwd(int32_t N, int32_t T, const int32_t* cu_seqlens, int32_t H, int32_t G, int32_t P, int32_t Ns,
                    int32_t dtype, int32_t softplus, const void* x, int64_t ldx, const float* dt, const float* A,
                    const void* B, int64_t ldb, const void* C, int64_t ldc, const float* D, const float* dt_bias,
                    const float* initial_state, const void* dy, const float* d_final_state, void* dx, float* ddt,
                    float* dA, void* dB, void* dC, float* dD, float* ddt_bias, float* d_initial_state, void* ws,
                    size_t ws_bytes, hipStream_t stream);

/* One token of N sequences: x [N, H, P], dt [N, H], B, C [N, G, Ns] and state
 * [N, H, P, Ns] into y [N, H, P] and state_out, which may be state itself. */
int qdelta_scan_step(int32_t N, int32_t H, int32_t G, int32_t P, int32_t Ns, int32_t dtype, int32_t softplus,
                     const void* x, int64_t ldx, const float* dt, const float* A, const void* B, int64_t ldb,
                     const void* C, int64_t ldc, const float* D, const float* dt_bias, const float* state,
                     float* state_out, void* y, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* QDELTA_MIXER_H */
