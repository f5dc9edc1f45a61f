// What the entry points share on the host: checks of layouts and workspaces, the status of a launch.
#pragma once
#pragma GCC visibility push(default)
#include "../../include/sla.h"
#pragma GCC visibility pop

#include "common.h"

namespace sla {

// A caller-given layout: rows of d contiguous channels, 16-byte aligned, at non-negative strides.
inline int make_layout(const void* base, const sla_strides* st, int H, int N, Layout* L) {
  if (!st) {
    *L = contiguous_layout(H, N);
    return SLA_OK;
  }
  if (st->batch < 0 || st->head < 0 || st->token < D) return SLA_ERR_LAYOUT;
  if ((st->batch | st->head | st->token) & 7) return SLA_ERR_LAYOUT;
  if ((uintptr_t)base & 15) return SLA_ERR_LAYOUT;
  L->sb = st->batch; L->sh = st->head; L->sn = st->token;
  return SLA_OK;
}

inline int check_ws(const void* ws, size_t bytes, size_t need) {
  if (!ws || ((uintptr_t)ws & 255) || bytes < need) return SLA_ERR_WORKSPACE;
  return SLA_OK;
}

inline int launch_status() { return hipGetLastError() == hipSuccess ? SLA_OK : SLA_ERR_HIP; }

// The entry points of rope.h, norm.h and xattn.h read and write sixteen bytes at a time in every layout.
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline int make_aligned_layout(const void* base, const sla_strides* st, int H, int N, Layout* L) {
  return aligned16(base) ? make_layout(base, st, H, N, L) : SLA_ERR_LAYOUT;
}

// A norm's eps as the kernels take it: a normal fp32 number above zero.
inline bool eps_ok(double eps) { return (float)eps >= 1.17549435e-38f && (float)eps <= 3.402823466e38f; }

}  // namespace sla
