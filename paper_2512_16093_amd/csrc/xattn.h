// Attention to a sequence of another length (k_xattn.hip): what its entry points hand to the kernels.
#pragma once
#include "common.h"

namespace sla {

// How a kernel's work is dealt out: workgroups of nw wavefronts, tiles of 32 nw rows of each slice (query rows, or keys for dk
// and dv), each tile's walk (over the keys, or over the steps of the queries) in `splits` pieces of `chunk`.
struct XattnDeal {
  int nw, tiles, splits, chunk;
};
struct XattnArgs {
  const bf16_t *q, *k, *v, *o, *dout;   // (o, dout: backward)
  bf16_t *out, *dq, *dk, *dv;
  float* lse;                           // forward: may be nullptr
  const float* lse_in;
  const int32_t* lens;                  // nullptr: Nk
  Layout lq, lk, lv, lo, ldo, ldq, ldk, ldv;   // (lo: of out or o)
  int B, H, G, Nq, Nk;                  // G: key heads
  int group, rows;                      // query heads of a key head; group * Nq: query rows of a key head, head after head
  float scale, c2;                      // c2 = scale * log2(e)
  XattnDeal fwd, dqd, dkv;
  // workspace
  float *part_o, *part_ml;              // forward: fp32 [splits, B H Nq, 128], [splits, B H Nq, 4]
  float *lse2, *neg_delta;                 // backward: fp32 [B H, padded_rows(Nq)]
  float *part_dq, *part_dk, *part_dv;   // fp32 [splits, ...]
};
__host__ __device__ inline int xattn_padded_rows(int Nq) { return (Nq + 63) / 64 * 64; }
XattnDeal xattn_deal_rows(int B, int G, int rows, int Nk, bool fwd);  // forward, or dq
XattnDeal xattn_deal_keys(int B, int G, int group, int Nq, int Nk);   // dk, dv
void launch_xattn_fwd(const XattnArgs& a, hipStream_t stream);
void launch_xattn_bwd(const XattnArgs& a, hipStream_t stream);

}  // namespace sla
