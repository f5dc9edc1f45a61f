// Kernels that work token by token (k_rope.hip, k_norm.hip): a team of threads per token, sixteen bytes a thread and turn.
#pragma once
#include "common.h"

namespace sla {

// Rotary positions, include/rope.h.  (turns, axis: rope_plan's)
struct RopeTurns {
  uint64_t turns[64];
  uint8_t axis[64];
};
struct RopeTensor {
  const bf16_t* x;    // the forward pass's input (backward without a norm: nullptr)
  const bf16_t* dy;   // backward: the output's gradient
  const bf16_t* w;    // nullptr: ones
  bf16_t* y;          // forward: the output; backward: the input's gradient
  float* part;        // backward: partial sums of the weight's gradient [workgroups, width]; nullptr: not wanted
  float* dw;
  Layout lx, ldy, ly;
  int H;              // 0: this tensor is not there
};
struct RopeArgs {
  RopeTensor t[2];    // q, k
  const int32_t* pos;
  long long pos_batch;
  int B, N;
  float eps;
  RopeTurns plan;
};
void launch_rope_fwd(const RopeArgs& a, int norm, bool halves, hipStream_t stream);
void launch_rope_bwd(const RopeArgs& a, int norm, bool halves, hipStream_t stream);
int rope_bwd_workgroups(long long tokens, int heads);   // of one tensor (heads: of the wider one)

// Root-mean-square norm, include/norm.h.
void launch_norm_fwd(const void* x, const void* res, const void* w, void* h, void* y, int M, int K, float eps, hipStream_t stream);
// h (res given) and r of every row
void launch_norm_stats(const void* x, const void* res, void* h, float* r, int M, int K, float eps, hipStream_t stream);
void launch_norm_bwd(const void* dy, const void* dh, const void* h, const void* w, void* dx, float* dw, float* part, int M, int K,
                     float eps, hipStream_t stream);
int norm_bwd_workgroups(int M, int K);

// dw[i][x] = sum over g < n_part of part[i][g][x], x < width[i], in a fixed order (i: blockIdx.y; part nullptr: nothing)
struct PartialSums {
  const float* part[2];
  float* dw[2];
  int width[2], n_part;
};
void launch_sum_partials(const PartialSums& s, hipStream_t stream);

// Sixteen (eight) bytes from and to memory; NT: past the caches.
template <bool NT, class V>
__device__ __forceinline__ V load_from(const bf16_t* p) {
  typedef int words __attribute__((ext_vector_type(sizeof(V) / 4)));
  if constexpr (NT) return __builtin_bit_cast(V, __builtin_nontemporal_load((const words*)p));
  else return *(const V*)p;
}
template <bool NT, class V>
__device__ __forceinline__ void store_to(bf16_t* p, const V& v) {
  typedef int words __attribute__((ext_vector_type(sizeof(V) / 4)));
  if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(words, v), (words*)p);
  else *(V*)p = v;
}
// A team of T threads (64: a wavefront, four teams to a workgroup; else the workgroup).  sum(): of one number per thread,
// to all of them; red: T / 64 floats of shared memory that the sum before the last one may still be read from (callers
// alternate between two).
template <int T>
__device__ __forceinline__ float team_sum(float x, float* red) {
  x = rows_sum(row_sum(x));
  if constexpr (T > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) red[w] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) x += red[i];
  }
  return x;
}

}  // namespace sla
