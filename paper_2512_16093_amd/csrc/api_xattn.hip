// C ABI of the attention to a sequence of another length (include/xattn.h): argument checks, the workspace, the launches.
#pragma GCC visibility push(default)
#include "../../include/xattn.h"
#pragma GCC visibility pop

#include <math.h>

#include "host.h"
#include "xattn.h"

using namespace sla;

namespace {

// Shapes and the scale, and how the work is dealt out.
int xattn_problem(int B, int H, int Hkv, int Nq, int Nk, int d, double scale, XattnArgs* a) {
  if (B < 1 || H < 1 || Hkv < 1 || Nq < 1 || Nk < 1 || d != D || H % Hkv || (long long)B * H > 65535) return SLA_ERR_SHAPE;
  if ((long long)B * H * Nq >= 1ll << 30 || (long long)B * Hkv * Nk >= 1ll << 30) return SLA_ERR_SHAPE;
  if (!(scale >= 0.0) || !(scale <= 1e30) || (scale > 0.0 && scale < 1e-30)) return SLA_ERR_VALUE;
  a->B = B; a->H = H; a->G = Hkv; a->Nq = Nq; a->Nk = Nk;
  a->group = H / Hkv;
  a->rows = a->group * Nq;
  a->scale = (float)(scale == 0.0 ? 1.0 / sqrt((double)D) : scale);
  a->c2 = (float)((scale == 0.0 ? 1.0 / sqrt((double)D) : scale) * 1.4426950408889634);
  a->fwd = xattn_deal_rows(B, Hkv, a->rows, Nk, true);
  a->dqd = xattn_deal_rows(B, Hkv, a->rows, Nk, false);
  a->dkv = xattn_deal_keys(B, Hkv, a->group, Nq, Nk);
  return SLA_OK;
}
// Lays the workspace out from `base` (nullptr: only its size).
size_t fwd_map(XattnArgs* a, unsigned char* base) {
  const size_t rows = (size_t)a->B * a->H * a->Nq;
  size_t o = 0;
  auto take = [&](size_t floats) { float* p = (float*)(base + o); o += align256(4 * floats); return p; };
  if (a->fwd.splits > 1) {
    a->part_o = take(a->fwd.splits * rows * D);
    a->part_ml = take(a->fwd.splits * rows * 4);
  }
  return o ? o : 256;
}
size_t bwd_map(XattnArgs* a, unsigned char* base) {
  const size_t rows = (size_t)a->B * a->H * a->Nq, keys = (size_t)a->B * a->G * a->Nk, padded = (size_t)a->B * a->H * xattn_padded_rows(a->Nq);
  size_t o = 0;
  auto take = [&](size_t floats) { float* p = (float*)(base + o); o += align256(4 * floats); return p; };
  a->lse2 = take(padded);
  a->neg_delta = take(padded);
  if (a->dqd.splits > 1) a->part_dq = take(a->dqd.splits * rows * D);
  if (a->dkv.splits > 1) {
    a->part_dk = take(a->dkv.splits * keys * D);
    a->part_dv = take(a->dkv.splits * keys * D);
  }
  return o;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t xattn_workspace_bytes(int B, int H, int Hkv, int Nq, int Nk, int d) {
  XattnArgs a{};
  return xattn_problem(B, H, Hkv, Nq, Nk, d, 0.0, &a) == SLA_OK ? fwd_map(&a, nullptr) : 0;
}

int xattn_fwd(const void* q, const void* k, const void* v, void* out, float* lse, const sla_strides* q_strides,
              const sla_strides* k_strides, const sla_strides* v_strides, const sla_strides* out_strides, const int32_t* k_lens,
              int B, int H, int Hkv, int Nq, int Nk, int d, double scale, void* workspace, size_t workspace_bytes,
              sla_stream_t stream) {
  if (!q || !k || !v || !out) return SLA_ERR_NULL;
  XattnArgs a{};
  int st;
  if ((st = xattn_problem(B, H, Hkv, Nq, Nk, d, scale, &a)) != SLA_OK) return st;
  if ((st = make_aligned_layout(q, q_strides, H, Nq, &a.lq)) != SLA_OK) return st;
  if ((st = make_aligned_layout(k, k_strides, Hkv, Nk, &a.lk)) != SLA_OK) return st;
  if ((st = make_aligned_layout(v, v_strides, Hkv, Nk, &a.lv)) != SLA_OK) return st;
  if ((st = make_aligned_layout(out, out_strides, H, Nq, &a.lo)) != SLA_OK) return st;
  if (((uintptr_t)lse & 3) || ((uintptr_t)k_lens & 3)) return SLA_ERR_LAYOUT;
  if ((st = check_ws(workspace, workspace_bytes, fwd_map(&a, (unsigned char*)workspace))) != SLA_OK) return st;
  a.q = (const bf16_t*)q; a.k = (const bf16_t*)k; a.v = (const bf16_t*)v;
  a.out = (bf16_t*)out;
  a.lse = lse;
  a.lens = k_lens;
  launch_xattn_fwd(a, (hipStream_t)stream);
  return launch_status();
}

size_t xattn_bwd_workspace_bytes(int B, int H, int Hkv, int Nq, int Nk, int d) {
  XattnArgs a{};
  return xattn_problem(B, H, Hkv, Nq, Nk, d, 0.0, &a) == SLA_OK ? bwd_map(&a, nullptr) : 0;
}

int xattn_bwd(const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse, void* dq, void* dk,
              void* dv, const xattn_bwd_strides* strides, const int32_t* k_lens, int B, int H, int Hkv, int Nq, int Nk, int d,
              double scale, void* workspace, size_t workspace_bytes, sla_stream_t stream) {
  if (!q || !k || !v || !out || !dout || !lse || !dq || !dk || !dv) return SLA_ERR_NULL;
  XattnArgs a{};
  int st;
  if ((st = xattn_problem(B, H, Hkv, Nq, Nk, d, scale, &a)) != SLA_OK) return st;
  static const xattn_bwd_strides contiguous = {};
  const xattn_bwd_strides& s = strides ? *strides : contiguous;
  if ((st = make_aligned_layout(q, s.q, H, Nq, &a.lq)) != SLA_OK) return st;
  if ((st = make_aligned_layout(k, s.k, Hkv, Nk, &a.lk)) != SLA_OK) return st;
  if ((st = make_aligned_layout(v, s.v, Hkv, Nk, &a.lv)) != SLA_OK) return st;
  if ((st = make_aligned_layout(out, s.out, H, Nq, &a.lo)) != SLA_OK) return st;
  if ((st = make_aligned_layout(dout, s.dout, H, Nq, &a.ldo)) != SLA_OK) return st;
  if ((st = make_aligned_layout(dq, s.dq, H, Nq, &a.ldq)) != SLA_OK) return st;
  if ((st = make_aligned_layout(dk, s.dk, Hkv, Nk, &a.ldk)) != SLA_OK) return st;
  if ((st = make_aligned_layout(dv, s.dv, Hkv, Nk, &a.ldv)) != SLA_OK) return st;
  if (((uintptr_t)lse & 3) || ((uintptr_t)k_lens & 3)) return SLA_ERR_LAYOUT;
  if ((st = check_ws(workspace, workspace_bytes, bwd_map(&a, (unsigned char*)workspace))) != SLA_OK) return st;
  a.q = (const bf16_t*)q; a.k = (const bf16_t*)k; a.v = (const bf16_t*)v;
  a.o = (const bf16_t*)out;
  a.dout = (const bf16_t*)dout;
  a.lse_in = lse;
  a.dq = (bf16_t*)dq; a.dk = (bf16_t*)dk; a.dv = (bf16_t*)dv;
  a.lens = k_lens;
  launch_xattn_bwd(a, (hipStream_t)stream);
  return launch_status();
}

}  // extern "C"
#pragma GCC visibility pop
