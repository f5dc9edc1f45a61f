/*
 * xattn.h -- C ABI of attention to a sequence of another length on MI355X (gfx950), part of
 * libsla.so: the cross attention of a DiT block, whose queries are the video's tokens and whose keys
 * and values are an encoder's states (a prompt, an image), in training and inference; and the same
 * for a few query tokens against a long memory.
 *
 *   out[n] = sum_t softmax_t(scale Q[n].K[t]) V[t]    over the first k_lens[b] of the Nk keys of sample b,
 *   lse[n] = log sum_t exp(scale Q[n].K[t])           (natural logarithm)
 *
 * Query heads may share key heads: head h of H reads head h / (H / Hkv) of Hkv.  A sample without keys
 * gives zeros and lse = -infinity.  What lies in keys and values behind k_lens[b] is not used, whatever it is
 * (NaN and infinities included); a NaN in a query or in a key that is used makes the rows that meet it NaN, in
 * out and in lse.
 * The products run in bf16 on the matrix cores with fp32 accumulation, softmax and its statistics in
 * fp32; the weights are rounded to bf16 for the product with V, and divided by the sum of the ROUNDED
 * weights; lse is that of the unrounded ones.
 * |scale Q.K| up to 2^24 is inside what the forward pass takes: fp32 does not resolve larger scores to a unit,
 * and from 2^31 / log2(e) on a row can come out NaN or as one without keys.  The backward pass forms its weights
 * anew from lse, which is rounded to fp32: they are off by up to 2^-22 |lse| of their size, within a rounding to
 * bf16 up to |lse| = 2^14.
 *
 * Rules as in sla.h: every tensor pointer is a DEVICE pointer owned by the caller, strides are HOST
 * structs; the library allocates nothing and never synchronises; work is enqueued on `stream`; scratch
 * lives in `workspace` (256-byte aligned, at least as many bytes as the function beside each entry
 * point says, contents undefined before and after; calls that share one must be stream-ordered); inputs are
 * never written; outputs must not alias inputs, each other or the workspace.  Returns SLA_OK or a negative
 * sla_status; argument errors are found on the host before any launch.  Results are deterministic (no
 * floating-point atomics).
 * Supported: d == 128; H a multiple of Hkv; Nq, Nk >= 1; B H <= 65535; B H Nq and B Hkv Nk below 2^30;
 * scale 0 (1 / sqrt(d)) or from 1e-30 to 1e30 (else SLA_ERR_VALUE); strides as for sla_attention_fwd_strided
 * (NULL = contiguous; 16-byte aligned bases in either case, else SLA_ERR_LAYOUT).
 */
#ifndef XATTN_H_
#define XATTN_H_

#include <stddef.h>
#include <stdint.h>

#include "sla.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Host-only.  Workspace bytes of xattn_fwd (partial results where few queries meet many keys); 0 if
 * the arguments are not supported. */
size_t xattn_workspace_bytes(int B, int H, int Hkv, int Nq, int Nk, int d);

/*   q       in   bf16 [B,H,Nq,d]
 *   k, v    in   bf16 [B,Hkv,Nk,d]
 *   out     out  bf16 [B,H,Nq,d]
 *   lse     out  fp32 [B,H,Nq], contiguous; NULL = not wanted (xattn_bwd needs it)
 *   k_lens  in   int32 [B]: keys of each sample (taken as 0 below 0, as Nk above Nk); NULL = all of them */
int xattn_fwd(const void* q, const void* k, const void* v, void* out, float* lse, const sla_strides* q_strides,
              const sla_strides* k_strides, const sla_strides* v_strides, const sla_strides* out_strides,
              const int32_t* k_lens, int B, int H, int Hkv, int Nq, int Nk, int d, double scale, void* workspace,
              size_t workspace_bytes, sla_stream_t stream);

/* Host-only.  Workspace bytes of xattn_bwd; 0 if the arguments are not supported. */
size_t xattn_bwd_workspace_bytes(int B, int H, int Hkv, int Nq, int Nk, int d);

/* A layout per tensor of the backward pass (HOST pointers; NULL = contiguous). */
typedef struct {
  const sla_strides *q, *k, *v, *out, *dout, *dq, *dk, *dv;
} xattn_bwd_strides;

/* Gradients, with P the weights (from lse) and delta[n] = dout[n].out[n]:
 *   dS = P o (dout V^T - delta),   dq = scale dS K,   dk = scale dS^T q,   dv = P^T dout;
 * dk and dv of a shared head are sums over its query heads, those of keys behind k_lens[b] are zero.
 *   q, k, v, k_lens, scale   in   as in the forward call
 *   out, lse    in   the forward call's
 *   dout        in   bf16 [B,H,Nq,d]   gradient of out
 *   dq, dk, dv  out  bf16, shaped like q, k, v */
int xattn_bwd(const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse, void* dq,
              void* dk, void* dv, const xattn_bwd_strides* strides, const int32_t* k_lens, int B, int H, int Hkv, int Nq,
              int Nk, int d, double scale, void* workspace, size_t workspace_bytes, sla_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* XATTN_H_ */
