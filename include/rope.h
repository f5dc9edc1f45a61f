/*
 * rope.h -- C ABI of rotary positions over several axes on MI355X (gfx950), part of libsla.so.
 *
 * The operation stands between a DiT block's QKV projection and its attention (sla.h): every token
 * of a video has a place on several axes (time, height, width), and each channel pair of a head is
 * turned by an angle proportional to the coordinate of ONE of them.  Queries and keys are commonly
 * normed on the way, and are here:
 *
 *   z  = x r o w,  r = 1 / sqrt(mean(x^2) + eps)    (ROPE_NORM_NONE: z = x)
 *        mean over the d channels of a head (ROPE_NORM_HEAD, w [d]) or over all heads' channels of
 *        a token (ROPE_NORM_TOKEN, w [H d], head after head);
 *   y_lo = z_lo cos a - z_hi sin a,   y_hi = z_lo sin a + z_hi cos a
 *        for the channel pairs j = 0 .. 63 = (2 j, 2 j + 1) (ROPE_INTERLEAVED) or (j, j + 64)
 *        (ROPE_HALVES); the first pairs[0] belong to axis 0, the next pairs[1] to axis 1, the rest
 *        to axis 2; pair number i of an axis of n turns by a = position theta^(-i / n).
 *
 * Everything is computed in fp32 and rounded once to bf16 (nearest even).  The angle is formed in
 * 64-bit fixed point (turns modulo 1), so that it is good at position 2^31 - 1 as well as at 1: its
 * error is below 2^-28 turns.
 *
 * With a norm the SUM of the squares that a mean is taken of has to stay within fp32 (|x| up to 1e17 is inside
 * for every number of heads): beyond, the heads or tokens concerned come out zero or NaN.  In the backward pass
 * the same holds of the sums of |x o w o g|.
 *
 * Rules as in sla.h: every tensor pointer is a DEVICE pointer owned by the caller; the plan and the
 * strides are HOST structs read during the call; the library allocates nothing and never
 * synchronises; work is enqueued on `stream`; inputs are never written; outputs must not alias
 * inputs, each other or the workspace.  Returns SLA_OK or a negative sla_status; argument errors are
 * found on the host before any launch.  Results are deterministic (no floating-point atomics).
 * Supported: d == 128; 1 <= H, Hk <= 64 (Hk: heads of k, which need not be those of q); B, N >= 1
 * with B N < 2^24; strides as for sla_attention_fwd_strided (NULL = [B,H,N,d] contiguous; 16-byte aligned bases
 * in either case, else SLA_ERR_LAYOUT).
 */
#ifndef ROPE_H_
#define ROPE_H_

#include <stddef.h>
#include <stdint.h>

#include "sla.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ROPE_INTERLEAVED = 0, ROPE_HALVES = 1 } rope_pairing;
typedef enum { ROPE_NORM_NONE = 0, ROPE_NORM_HEAD = 1, ROPE_NORM_TOKEN = 2 } rope_norm;

/* How far every channel pair turns per step of its axis; filled by rope_make_plan, otherwise opaque. */
typedef struct {
  int32_t made, pairing;
  uint64_t turns[64]; /* turns per step, as a fraction of 2^64 */
  uint8_t axis[64];
} rope_plan;

/* Host-only.  pairs: channel pairs of each axis (none negative, together 64; an axis may have none);
 * theta: base of each axis, 1 <= theta <= 1e12.  SLA_ERR_NULL, SLA_ERR_SHAPE (pairs), SLA_ERR_VALUE
 * (theta) or SLA_ERR_UNSUPPORTED (pairing). */
int rope_make_plan(const int32_t pairs[3], const double theta[3], int pairing, rope_plan* plan);

/* q and k as the attention takes them.
 *   q, k             in   bf16 [B,H,N,d], [B,Hk,N,d] at q_strides, k_strides; k NULL: q alone (then
 *                         k_out is NULL too)
 *   positions        in   int32 [N,3] (positions_batch 0: every sample has the same) or [B,N,3] with
 *                         positions_batch int32 from one sample to the next (>= 3 N); any values
 *   q_weight, k_weight  in  bf16 [d] or [H d] / [Hk d] (see norm), 16-byte aligned; NULL = ones; not
 *                         read without a norm
 *   eps              added to the mean square: > 0 (not read without a norm)
 *   q_out, k_out     out  bf16, at q_out_strides, k_out_strides
 * SLA_ERR_UNSUPPORTED: norm not a rope_norm, or a plan that rope_make_plan did not make. */
int rope_qk_fwd(const void* q, const void* k, void* q_out, void* k_out, const sla_strides* q_strides,
                const sla_strides* k_strides, const sla_strides* q_out_strides, const sla_strides* k_out_strides,
                const int32_t* positions, int64_t positions_batch, const void* q_weight, const void* k_weight,
                int norm, double eps, int B, int H, int Hk, int N, int d, const rope_plan* plan, sla_stream_t stream);

/* Host-only.  Workspace bytes of rope_qk_bwd (partial sums of the weights' gradients); 0 if the
 * arguments are not supported. */
size_t rope_bwd_workspace_bytes(int B, int H, int Hk, int N, int d, int norm);

/* A layout per tensor of the backward pass (HOST pointers; NULL = contiguous). */
typedef struct {
  const sla_strides *dq_out, *dk_out, *q, *k, *dq, *dk;
} rope_bwd_strides;

/* Gradients of rope_qk_fwd: with g the gradient of the outputs turned back,
 *   dx = r (w o g) - x r^3 mean(x o w o g),   dw = sum g o x r over every token (and head, for w [d]).
 *   dq_out, dk_out   in   bf16   gradients of q_out and k_out (dk_out NULL: q alone)
 *   q, k             in   bf16   the forward pass's inputs (not read without a norm: may be NULL)
 *   dq, dk           out  bf16
 *   dq_weight, dk_weight  out  fp32 [d] or [H d] / [Hk d]; NULL = not wanted (must be NULL without a norm)
 *   workspace        256-byte aligned, rope_bwd_workspace_bytes(...) bytes; needed only where a
 *                    weight's gradient is wanted (else it may be NULL) */
int rope_qk_bwd(const void* dq_out, const void* dk_out, const void* q, const void* k, void* dq, void* dk,
                float* dq_weight, float* dk_weight, const rope_bwd_strides* strides, const int32_t* positions,
                int64_t positions_batch, const void* q_weight, const void* k_weight, int norm, double eps, int B,
                int H, int Hk, int N, int d, const rope_plan* plan, void* workspace, size_t workspace_bytes,
                sla_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* ROPE_H_ */
