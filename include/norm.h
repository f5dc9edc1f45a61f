/*
 * norm.h -- C ABI of the root-mean-square norm with the residual's addition on MI355X (gfx950),
 * part of libsla.so.
 *
 * The norm of the residual stream that a transformer block starts each of its parts with, and the
 * addition of the last part's result to that stream, in one pass over the data:
 *
 *   h = x + res, rounded to bf16 (the stream as it is stored; without res: h = x);
 *   y = h r o w,  r = 1 / sqrt(mean(h^2) + eps) over the K features, in fp32, rounded once to bf16.
 *
 * The norm is that of the STORED stream, so that norm_rms_bwd, which finds the stored one, gives the
 * gradient of exactly this function (the rounding of h passes gradients on unchanged).
 * w8a8_norm_linear_fwd (w8a8.h) is the same norm in front of a W8A8 Linear layer, y as 8-bit codes.
 *
 * Rules as in sla.h: every tensor pointer is a DEVICE pointer owned by the caller; the library
 * allocates nothing and never synchronises; work is enqueued on `stream`; inputs are never written;
 * outputs must not alias inputs, each other or the workspace.  Returns SLA_OK or a negative
 * sla_status; argument errors are found on the host before any launch.  Results are deterministic
 * (no floating-point atomics).
 * Tensors are bf16 [M, K], row-major and contiguous, 16-byte aligned (else SLA_ERR_LAYOUT).
 * Values are expected finite, and the sum of a row's squares within fp32 (|h| up to 1e17 is inside for every K):
 * beyond, that row alone comes out zero or NaN.  In the backward pass the same holds of the sum of |h o w o dy|.
 * Supported: K a multiple of 8, 8 <= K <= 16384; 1 <= M <= 2^22; eps > 0 (else SLA_ERR_VALUE).
 */
#ifndef NORM_H_
#define NORM_H_

#include <stddef.h>
#include <stdint.h>

#include "sla.h"

#ifdef __cplusplus
extern "C" {
#endif

/*   x    in   bf16 [M, K]
 *   res  in   bf16 [M, K]; NULL = none (then h is NULL too)
 *   w    in   bf16 [K]; NULL = ones
 *   h    out  bf16 [M, K]   x + res
 *   y    out  bf16 [M, K] */
int norm_rms_fwd(const void* x, const void* res, const void* w, void* h, void* y, int M, int K, double eps,
                 sla_stream_t stream);

/* Host-only.  Workspace bytes of norm_rms_bwd (partial sums of dw); 0 if the arguments are not supported. */
size_t norm_bwd_workspace_bytes(int M, int K);

/* Gradients: dx = dh + r (w o dy) - h r^3 mean(h o w o dy) (of x and of res alike), dw = sum over the
 * rows of dy o h r.
 *   dy   in   bf16 [M, K]   gradient of y
 *   dh   in   bf16 [M, K]   gradient that h has from elsewhere (the stream's further way); NULL = none
 *   h    in   bf16 [M, K]   the stored stream (the forward pass's h, or x)
 *   w    in   bf16 [K]; NULL = ones
 *   dx   out  bf16 [M, K]
 *   dw   out  fp32 [K]; NULL = not wanted
 *   workspace  256-byte aligned; needed only where dw is wanted (else it may be NULL) */
int norm_rms_bwd(const void* dy, const void* dh, const void* h, const void* w, void* dx, float* dw, int M, int K,
                 double eps, void* workspace, size_t workspace_bytes, sla_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* NORM_H_ */
