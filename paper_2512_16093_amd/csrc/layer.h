// Layer norm with gate and modulation (include/norm.h): what its entry points and those of the 4-bit layers (include/mxfp4.h)
// check on the host and hand to the kernels (k_layer.hip).
#pragma once
#pragma GCC visibility push(default)
#include "../../include/norm.h"
#pragma GCC visibility pop

#include "host.h"
#include "rows.h"

namespace sla {

struct SampleVec {
  const float* v;       // nullptr: not there
  long long stride;     // floats from one sample's to the next's
};
struct LayerArgs {
  const bf16_t *x, *res, *w, *b;
  SampleVec gate, scale, shift;
  bf16_t *h, *y;
  uint8_t *codes, *exps;   // the quantised rows of k_mxfp4.hip instead of y
  int M, K, rows;
  float eps;
};
struct LayerBwdArgs {
  const bf16_t *dy, *dh, *h, *res, *w, *b;
  SampleVec gate, scale;
  bf16_t *dx, *dres;
  norm_layer_grads grads;
  float* ws;
  int M, K, rows;
  float eps;
};
void launch_layer_fwd(const LayerArgs& a, hipStream_t stream);
void launch_layer_bwd(const LayerBwdArgs& a, hipStream_t stream);
size_t layer_bwd_bytes(int M, int K, int rows);

inline bool norm_dims_ok(int M, int K) { return M >= 1 && M <= (1 << 22) && K >= 8 && K <= 16384 && !(K & 7); }

inline int sample_vec(const float* v, int64_t stride, SampleVec* out) {
  *out = SampleVec{v, stride};
  return v && (!aligned16(v) || stride < 0 || (stride & 3)) ? SLA_ERR_LAYOUT : SLA_OK;
}
// The forward direction's arguments (y, or what stands in its place, is the caller's to check).
inline int layer_args(const void* x, const void* res, const void* w, const void* b, const norm_modulation* mod, void* h, int M,
                      int K, double eps, LayerArgs* a) {
  if (!x || !res != !h || (mod && mod->gate && !res)) return SLA_ERR_NULL;
  if (!norm_dims_ok(M, K) || (mod && mod->rows < 1)) return SLA_ERR_SHAPE;
  if (!eps_ok(eps)) return SLA_ERR_VALUE;
  if (!aligned16(x) || !aligned16(res) || !aligned16(w) || !aligned16(b) || !aligned16(h)) return SLA_ERR_LAYOUT;
  *a = LayerArgs{};
  if (mod) {
    if (int st = sample_vec(mod->gate, mod->gate_stride, &a->gate)) return st;
    if (int st = sample_vec(mod->scale, mod->scale_stride, &a->scale)) return st;
    if (int st = sample_vec(mod->shift, mod->shift_stride, &a->shift)) return st;
  }
  a->x = (const bf16_t*)x;
  a->res = (const bf16_t*)res;
  a->w = (const bf16_t*)w;
  a->b = (const bf16_t*)b;
  a->h = (bf16_t*)h;
  a->M = M;
  a->K = K;
  a->rows = mod ? mod->rows : M;
  a->eps = (float)eps;
  return SLA_OK;
}

}  // namespace sla
