/*
 * norm.h -- C ABI of the norms of the residual stream, with the residual's addition, on MI355X (gfx950),
 * part of libsla.so: the root-mean-square norm (norm_rms_*) and, below it, the layer norm with a sample's
 * modulation (norm_layer_*).
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

/* ---- Layer norm, gated and modulated ----
 *
 * What a block whose parts are steered by a timestep does between them: the last part's result joins the
 * stream through a gate, the stream is normed, and the normed rows are scaled and shifted, with gate, scale
 * and shift one vector per SAMPLE (`rows` consecutive rows):
 *
 *   h = x + gate o res, rounded to bf16 (without gate: x + res; without res: h = x);
 *   n = (h - mean(h)) r,  r = 1 / sqrt(mean((h - mean(h))^2) + eps)  over the K features;
 *   y = (n o w + b) o (1 + scale) + shift,  in fp32, rounded once to bf16.
 *
 * As above the norm is that of the STORED stream.  Mean and variance are two passes over a row that is held in
 * registers, so a mean that is large against the deviations costs no precision beyond that of h itself.
 * mxfp4_norm_linear_fwd (mxfp4.h) is the same norm in front of a 4-bit Linear layer.
 *
 * A row whose values are not finite, or whose sum of squared deviations is beyond fp32 (|h| up to 1e17 is inside
 * for every K), comes out NaN or zero, that row alone; in the backward pass the sums over rows then are NaN too.
 * Supported: as above; rows >= 1 (samples: M / rows, the last one may be shorter); the vectors of gate, scale and shift
 * are contiguous fp32 at 16-byte aligned bases and strides that are multiples of 4 and not negative (0: every sample has the same). */
typedef struct {
  const float *gate, *scale, *shift;                    /* DEVICE pointers, each [samples] vectors of K; NULL = none (1, 0, 0) */
  int64_t gate_stride, scale_stride, shift_stride;      /* floats from one sample's vector to the next's */
  int32_t rows;                                         /* rows per sample */
} norm_modulation;

/*   x    in   bf16 [M, K]
 *   res  in   bf16 [M, K]; NULL = none (then h is NULL too, and there is no gate: SLA_ERR_NULL)
 *   w, b in   bf16 [K]; NULL = ones, zeros
 *   mod  in   HOST struct read during the call; NULL = no gate, scale or shift
 *   h    out  bf16 [M, K]
 *   y    out  bf16 [M, K] */
int norm_layer_fwd(const void* x, const void* res, const void* w, const void* b, const norm_modulation* mod, void* h, void* y,
                   int M, int K, double eps, sla_stream_t stream);

/* Where the gradients of the vectors go; NULL = not wanted.  fp32, 16-byte aligned. */
typedef struct {
  float *w, *b;                                         /* [K] */
  float *gate, *scale, *shift;                          /* [samples, K], contiguous */
} norm_layer_grads;

/* Host-only.  Workspace bytes of norm_layer_bwd (partial sums); 0 if the arguments are not supported.
 * rows: per sample (M without a modulation). */
size_t norm_layer_bwd_workspace_bytes(int M, int K, int rows);

/* Gradients: with g = dy o (1 + scale) o w,
 *   dx = dh + r (g - mean(g) - n mean(g o n)),   dres = gate o dx,
 *   dw = sum dy o (1 + scale) o n,   db = sum dy o (1 + scale)      over all rows,
 *   dgate = sum dx o res,   dscale = sum dy o (n o w + b),   dshift = sum dy      over a sample's rows,
 * the sums in fp32, of dx before it is rounded.
 *   dy   in   bf16 [M, K]   gradient of y
 *   dh   in   bf16 [M, K]   gradient that h has from elsewhere (the stream's further way); NULL = none
 *   h    in   bf16 [M, K]   the stored stream (the forward pass's h, or x)
 *   res  in   bf16 [M, K]   needed only for the gate's gradient (else it may be NULL)
 *   w, b, mod  in           as in the forward call (b: needed only for the scale's gradient; shift is not read)
 *   dx   out  bf16 [M, K]   gradient of x (and of res, where there is no gate)
 *   dres out  bf16 [M, K]; NULL = not wanted (there has to be a gate, else SLA_ERR_NULL)
 *   grads out               HOST struct read during the call; NULL = none wanted
 *   workspace  256-byte aligned; needed only where a vector's gradient is wanted (else it may be NULL) */
int norm_layer_bwd(const void* dy, const void* dh, const void* h, const void* res, const void* w, const void* b,
                   const norm_modulation* mod, void* dx, void* dres, const norm_layer_grads* grads, int M, int K, double eps,
                   void* workspace, size_t workspace_bytes, sla_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* NORM_H_ */
