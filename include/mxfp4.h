/*
 * mxfp4.h -- C ABI of microscaled 4-bit floating point on MI355X (gfx950), part of libsla.so: a matrix
 * quantised to it, and the Linear layer whose weights and activations are both held in it, which runs on the
 * matrix cores at twice the rate of 8-bit operands.
 *
 * Format (the MXFP4 of the OCP Microscaling specification).  Along a row, every 32 consecutive features are
 * a block (the last one of a row may be shorter); a block has an 8-bit exponent E that stands for 2^(E - 127), and
 * each feature a 4-bit code, sign, two bits of exponent and one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 * negatives (codes 0..7, 8..15).  The feature is code times 2^(E - 127); E = 255 makes a whole block NaN.
 *
 * Quantisation of a block whose largest magnitude is m:
 *   E = floor(log2 m) - 2 + 127, at least 1: the quotients x / 2^(E - 127) lie below 8;
 *   code = the value nearest to the quotient, ties to the even code, 6 from 5 on (quotients between 6 and 8 are cut to 6).
 * A block that holds an infinity or a NaN becomes NaN (E = 255, codes 0).  E is at least 1, so that blocks whose
 * largest magnitude is below 2^-124 are rounded to multiples of 2^-127.
 *
 * The layer, for activations X [M, K] and weights W [N, K], each as its codes stand for it:
 *   Y[m, n] = sum_k X[m, k] W[n, k]  (+ bias[n]),  accumulated in fp32, rounded once to bf16.
 * Products of two codes are exact; the matrix cores add them up in fp32.
 *
 * A quantised matrix is an opaque OBJECT of mxfp4_bytes(R, K) bytes (codes in the order the matrix cores take
 * them, then the exponents), the same for weights and activations; mxfp4_pack and mxfp4_unpack turn it from and
 * into plain rows.  It is valid for this library version only.
 *
 * Rules as in sla.h: every tensor pointer is a DEVICE pointer owned by the caller; the library allocates
 * nothing and never synchronises; work is enqueued on `stream`; inputs are never written; outputs must not alias
 * inputs, each other or the workspace.  Objects and workspaces are 256-byte aligned and at least as large as the function
 * beside them says, else SLA_ERR_WORKSPACE; bf16 matrices are row-major, contiguous and 16-byte aligned (else
 * SLA_ERR_LAYOUT).  Returns SLA_OK or a negative sla_status; argument errors are found on the host before any launch.
 * Results are deterministic.
 * Supported: K and N multiples of 8 from 8 to 65536; 1 <= M, R <= 2^22 (R of a weight: N).
 */
#ifndef MXFP4_H_
#define MXFP4_H_

#include <stddef.h>
#include <stdint.h>

#include "norm.h"
#include "sla.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Host-only.  Bytes of the object of an [R, K] matrix; 0 if R or K is not supported. */
size_t mxfp4_bytes(int R, int K);

/* q = the object of x, bf16 [R, K]. */
int mxfp4_quantize(const void* x, int R, int K, void* q, size_t q_bytes, sla_stream_t stream);

/* x = what the codes of q stand for, bf16 [R, K] (exact; beyond the range of bf16 an infinity). */
int mxfp4_dequantize(const void* q, size_t q_bytes, int R, int K, void* x, sla_stream_t stream);

/* From and into plain rows (any alignment):
 *   codes      uint8 [R, K / 2]: features 2 i (low half) and 2 i + 1
 *   exponents  uint8 [R, ceil(K / 32)]
 * mxfp4_unpack: either output may be NULL. */
int mxfp4_pack(const uint8_t* codes, const uint8_t* exponents, int R, int K, void* q, size_t q_bytes, sla_stream_t stream);
int mxfp4_unpack(const void* q, size_t q_bytes, int R, int K, uint8_t* codes, uint8_t* exponents, sla_stream_t stream);

/* y = the layer of two objects.
 *   xq    in   object of the activations [M, K]
 *   wq    in   object of the weight [N, K]
 *   bias  in   bf16 [N], 16-byte aligned; NULL = none
 *   y     out  bf16 [M, N] */
int mxfp4_gemm_fwd(const void* xq, size_t xq_bytes, const void* wq, size_t wq_bytes, const void* bias, void* y, int M, int N,
                   int K, sla_stream_t stream);

/* The same of x, bf16 [M, K], quantised on the way (into the workspace, of mxfp4_bytes(M, K) bytes, whose contents are undefined
 * afterwards; calls that share one must be stream-ordered). */
int mxfp4_linear_fwd(const void* x, const void* wq, size_t wq_bytes, const void* bias, void* y, int M, int N, int K,
                     void* workspace, size_t workspace_bytes, sla_stream_t stream);

/* ---- The norm in front of the layer ----
 *
 * The layer norm of norm.h (norm_layer_fwd: x, res, w, b, mod, h, eps as there, K <= 16384), its result quantised instead of
 * stored: the same codes as mxfp4_quantize gives of norm_layer_fwd's y, which is not written. */
int mxfp4_norm_quantize(const void* x, const void* res, const void* w, const void* b, const norm_modulation* mod, void* h,
                        void* q, size_t q_bytes, int M, int K, double eps, sla_stream_t stream);
/* ... and the layer of it; workspace as for mxfp4_linear_fwd. */
int mxfp4_norm_linear_fwd(const void* x, const void* res, const void* norm_w, const void* norm_b, const norm_modulation* mod,
                          void* h, const void* wq, size_t wq_bytes, const void* bias, void* y, int M, int N, int K, double eps,
                          void* workspace, size_t workspace_bytes, sla_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* MXFP4_H_ */
