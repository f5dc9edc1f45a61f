// C ABI of the rotary positions (include/rope.h) and of the norms (include/norm.h): argument checks and the launch sequence.
#pragma GCC visibility push(default)
#include "../../include/norm.h"
#include "../../include/rope.h"
#pragma GCC visibility pop

#include <math.h>
#include <string.h>

#include "host.h"
#include "layer.h"
#include "rows.h"

using namespace sla;

namespace {

constexpr int32_t PLAN_MADE = 0x524F5045;

bool rope_dims_ok(int B, int H, int Hk, int N, int d) {
  return B >= 1 && N >= 1 && H >= 1 && H <= 64 && Hk >= 0 && Hk <= 64 && d == D && (long long)B * N < (1ll << 24);
}
// what forward and backward check of norm, plan and positions, and hand to the kernels
int rope_args(const int32_t* positions, int64_t positions_batch, const void* qw, const void* kw, int norm, double eps, int B, int N,
              const rope_plan* plan, RopeArgs* a) {
  if (norm < ROPE_NORM_NONE || norm > ROPE_NORM_TOKEN || plan->made != PLAN_MADE) return SLA_ERR_UNSUPPORTED;
  if (norm != ROPE_NORM_NONE && !eps_ok(eps)) return SLA_ERR_VALUE;
  if (((uintptr_t)positions & 3) || (positions_batch != 0 && positions_batch < 3ll * N)) return SLA_ERR_LAYOUT;
  if (norm != ROPE_NORM_NONE) {
    if (!aligned16(qw) || !aligned16(kw)) return SLA_ERR_LAYOUT;
    a->t[0].w = (const bf16_t*)qw;
    a->t[1].w = (const bf16_t*)kw;
  }
  a->pos = positions;
  a->pos_batch = positions_batch;
  a->B = B;
  a->N = N;
  a->eps = norm != ROPE_NORM_NONE ? (float)eps : 0.f;
  memcpy(a->plan.turns, plan->turns, sizeof(plan->turns));
  memcpy(a->plan.axis, plan->axis, sizeof(plan->axis));
  return SLA_OK;
}
size_t rope_width(int heads, int norm) { return norm == ROPE_NORM_HEAD ? D : (size_t)heads * D; }
size_t part_bytes(long long tokens, int heads_max, int heads, int norm) {
  return align256((size_t)rope_bwd_workgroups(tokens, heads_max) * rope_width(heads, norm) * 4);
}
}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int rope_make_plan(const int32_t pairs[3], const double theta[3], int pairing, rope_plan* plan) {
  if (!pairs || !theta || !plan) return SLA_ERR_NULL;
  long long sum = 0;
  for (int i = 0; i < 3; ++i) {
    if (pairs[i] < 0) return SLA_ERR_SHAPE;
    sum += pairs[i];
  }
  if (sum != D / 2) return SLA_ERR_SHAPE;
  for (int i = 0; i < 3; ++i)
    if (!(theta[i] >= 1.0 && theta[i] <= 1e12)) return SLA_ERR_VALUE;
  if (pairing != ROPE_INTERLEAVED && pairing != ROPE_HALVES) return SLA_ERR_UNSUPPORTED;
  const long double turn = 6.283185307179586476925286766559005768L;
  int j = 0;
  for (int ax = 0; ax < 3; ++ax) {
    const int n = pairs[ax];
    // theta^(-i / n) from the i-th root's powers, by squaring: 64 bits each, at most 2^-58 off in the last of 64
    long double power[D / 2] = {1.0L};
    const long double root = n > 1 ? powl((long double)theta[ax], -1.0L / n) : 1.0L;
    for (int i = 1; i < n; ++i) power[i] = power[i / 2] * power[i / 2] * ((i & 1) ? root : 1.0L);
    for (int i = 0; i < n; ++i, ++j) {
      plan->turns[j] = (uint64_t)(power[i] / turn * 18446744073709551616.0L + 0.5L);   // (at most 1 / 2 pi: below one turn a step)
      plan->axis[j] = (uint8_t)ax;
    }
  }
  plan->pairing = pairing;
  plan->made = PLAN_MADE;
  return SLA_OK;
}

int rope_qk_fwd(const void* q, const void* k, void* q_out, void* k_out, const sla_strides* q_strides,
                const sla_strides* k_strides, const sla_strides* q_out_strides, const sla_strides* k_out_strides,
                const int32_t* positions, int64_t positions_batch, const void* q_weight, const void* k_weight, int norm,
                double eps, int B, int H, int Hk, int N, int d, const rope_plan* plan, sla_stream_t stream) {
  if (!q || !q_out || !k != !k_out || !positions || !plan) return SLA_ERR_NULL;
  if (!rope_dims_ok(B, H, Hk, N, d) || (k && Hk < 1)) return SLA_ERR_SHAPE;
  RopeArgs a{};
  if (int st = rope_args(positions, positions_batch, q_weight, k ? k_weight : nullptr, norm, eps, B, N, plan, &a)) return st;
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const sla_strides* is[2] = {q_strides, k_strides};
  const sla_strides* os[2] = {q_out_strides, k_out_strides};
  for (int i = 0; i < (k ? 2 : 1); ++i) {
    const int heads = i ? Hk : H;
    if (int st = make_aligned_layout(in[i], is[i], heads, N, &a.t[i].lx)) return st;
    if (int st = make_aligned_layout(out[i], os[i], heads, N, &a.t[i].ly)) return st;
    a.t[i].x = (const bf16_t*)in[i];
    a.t[i].y = (bf16_t*)out[i];
    a.t[i].H = heads;
  }
  launch_rope_fwd(a, norm, plan->pairing == ROPE_HALVES, (hipStream_t)stream);
  return launch_status();
}

size_t rope_bwd_workspace_bytes(int B, int H, int Hk, int N, int d, int norm) {
  if (!rope_dims_ok(B, H, Hk, N, d) || norm < ROPE_NORM_NONE || norm > ROPE_NORM_TOKEN) return 0;
  if (norm == ROPE_NORM_NONE) return 256;
  const int most = H > Hk ? H : Hk;
  return part_bytes((long long)B * N, most, H, norm) + (Hk ? part_bytes((long long)B * N, most, Hk, norm) : 0);
}

int rope_qk_bwd(const void* dq_out, const void* dk_out, const void* q, const void* k, void* dq, void* dk, float* dq_weight,
                float* dk_weight, const rope_bwd_strides* strides, const int32_t* positions, int64_t positions_batch,
                const void* q_weight, const void* k_weight, int norm, double eps, int B, int H, int Hk, int N, int d,
                const rope_plan* plan, void* workspace, size_t workspace_bytes, sla_stream_t stream) {
  const bool with_k = dk_out != nullptr, normed = norm != ROPE_NORM_NONE;
  if (!dq_out || !dq || !dk_out != !dk || !positions || !plan) return SLA_ERR_NULL;
  if (normed && (!q || (with_k && !k))) return SLA_ERR_NULL;
  if ((dq_weight || dk_weight) && !normed) return SLA_ERR_UNSUPPORTED;
  if (dk_weight && !with_k) return SLA_ERR_NULL;
  if (!rope_dims_ok(B, H, Hk, N, d) || (with_k && Hk < 1)) return SLA_ERR_SHAPE;
  const int hk = with_k ? Hk : 0;
  RopeArgs a{};
  if (int st = rope_args(positions, positions_batch, q_weight, with_k ? k_weight : nullptr, norm, eps, B, N, plan, &a)) return st;
  static const rope_bwd_strides contiguous = {};
  const rope_bwd_strides& s = strides ? *strides : contiguous;
  const void *dy[2] = {dq_out, dk_out}, *x[2] = {q, k};
  void* dx[2] = {dq, dk};
  float* dw[2] = {dq_weight, dk_weight};
  const sla_strides *ds[2] = {s.dq_out, s.dk_out}, *xs[2] = {s.q, s.k}, *gs[2] = {s.dq, s.dk};
  const int most = H > hk ? H : hk;
  unsigned char* ws = (unsigned char*)workspace;
  for (int i = 0; i < (with_k ? 2 : 1); ++i) {
    const int heads = i ? hk : H;
    RopeTensor& t = a.t[i];
    if (int st = make_aligned_layout(dy[i], ds[i], heads, N, &t.ldy)) return st;
    if (normed)
      if (int st = make_aligned_layout(x[i], xs[i], heads, N, &t.lx)) return st;
    if (int st = make_aligned_layout(dx[i], gs[i], heads, N, &t.ly)) return st;
    t.dy = (const bf16_t*)dy[i];
    t.x = normed ? (const bf16_t*)x[i] : nullptr;
    t.y = (bf16_t*)dx[i];
    t.H = heads;
    t.dw = dw[i];
    t.part = dw[i] ? (float*)ws : nullptr;
    if ((uintptr_t)dw[i] & 3) return SLA_ERR_LAYOUT;
    ws += part_bytes((long long)B * N, most, heads, norm);
  }
  if (dq_weight || dk_weight)
    if (int st = check_ws(workspace, workspace_bytes, rope_bwd_workspace_bytes(B, H, hk, N, d, norm))) return st;
  launch_rope_bwd(a, norm, plan->pairing == ROPE_HALVES, (hipStream_t)stream);
  return launch_status();
}

int norm_rms_fwd(const void* x, const void* res, const void* w, void* h, void* y, int M, int K, double eps,
                 sla_stream_t stream) {
  if (!x || !y || !res != !h) return SLA_ERR_NULL;
  if (!norm_dims_ok(M, K)) return SLA_ERR_SHAPE;
  if (!eps_ok(eps)) return SLA_ERR_VALUE;
  if (!aligned16(x) || !aligned16(res) || !aligned16(w) || !aligned16(h) || !aligned16(y)) return SLA_ERR_LAYOUT;
  launch_norm_fwd(x, res, w, h, y, M, K, (float)eps, (hipStream_t)stream);
  return launch_status();
}

size_t norm_bwd_workspace_bytes(int M, int K) {
  return norm_dims_ok(M, K) ? align256((size_t)norm_bwd_workgroups(M, K) * K * 4) : 0;
}

int norm_rms_bwd(const void* dy, const void* dh, const void* h, const void* w, void* dx, float* dw, int M, int K, double eps,
                 void* workspace, size_t workspace_bytes, sla_stream_t stream) {
  if (!dy || !h || !dx) return SLA_ERR_NULL;
  if (!norm_dims_ok(M, K)) return SLA_ERR_SHAPE;
  if (!eps_ok(eps)) return SLA_ERR_VALUE;
  if (dw)
    if (int st = check_ws(workspace, workspace_bytes, norm_bwd_workspace_bytes(M, K))) return st;
  if (!aligned16(dy) || !aligned16(dh) || !aligned16(h) || !aligned16(w) || !aligned16(dx) || ((uintptr_t)dw & 3)) return SLA_ERR_LAYOUT;
  launch_norm_bwd(dy, dh, h, w, dx, dw, (float*)workspace, M, K, (float)eps, (hipStream_t)stream);
  return launch_status();
}

int norm_layer_fwd(const void* x, const void* res, const void* w, const void* b, const norm_modulation* mod, void* h, void* y,
                   int M, int K, double eps, sla_stream_t stream) {
  if (!y) return SLA_ERR_NULL;
  LayerArgs a;
  if (int st = layer_args(x, res, w, b, mod, h, M, K, eps, &a)) return st;
  if (!aligned16(y)) return SLA_ERR_LAYOUT;
  a.y = (bf16_t*)y;
  launch_layer_fwd(a, (hipStream_t)stream);
  return launch_status();
}

size_t norm_layer_bwd_workspace_bytes(int M, int K, int rows) {
  return norm_dims_ok(M, K) && rows >= 1 ? layer_bwd_bytes(M, K, rows) : 0;
}

int norm_layer_bwd(const void* dy, const void* dh, const void* h, const void* res, const void* w, const void* b,
                   const norm_modulation* mod, void* dx, void* dres, const norm_layer_grads* grads, int M, int K, double eps,
                   void* workspace, size_t workspace_bytes, sla_stream_t stream) {
  static const norm_layer_grads none = {};
  const norm_layer_grads& g = grads ? *grads : none;
  const bool gated = mod && mod->gate;
  if (!dy || !h || !dx || (dres && !gated) || (g.gate && (!gated || !res))) return SLA_ERR_NULL;
  if (!norm_dims_ok(M, K) || (mod && mod->rows < 1)) return SLA_ERR_SHAPE;
  if (!eps_ok(eps)) return SLA_ERR_VALUE;
  const int rows = mod ? mod->rows : M;
  if (g.w || g.b || g.gate || g.scale || g.shift)
    if (int st = check_ws(workspace, workspace_bytes, layer_bwd_bytes(M, K, rows))) return st;
  const void* const all[] = {dy, dh, h, res, w, b, dx, dres, g.w, g.b, g.gate, g.scale, g.shift};
  for (const void* p : all)
    if (!aligned16(p)) return SLA_ERR_LAYOUT;
  LayerBwdArgs a{};
  if (mod) {
    if (int st = sample_vec(mod->gate, mod->gate_stride, &a.gate)) return st;
    if (int st = sample_vec(mod->scale, mod->scale_stride, &a.scale)) return st;
  }
  a.dy = (const bf16_t*)dy;
  a.dh = (const bf16_t*)dh;
  a.h = (const bf16_t*)h;
  a.res = g.gate ? (const bf16_t*)res : nullptr;
  a.w = (const bf16_t*)w;
  a.b = (const bf16_t*)b;
  a.dx = (bf16_t*)dx;
  a.dres = (bf16_t*)dres;
  a.grads = g;
  a.ws = (float*)workspace;
  a.M = M;
  a.K = K;
  a.rows = rows;
  a.eps = (float)eps;
  launch_layer_bwd(a, (hipStream_t)stream);
  return launch_status();
}

}  // extern "C"
#pragma GCC visibility pop
