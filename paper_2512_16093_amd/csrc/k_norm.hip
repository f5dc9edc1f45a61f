// Root-mean-square norm with the residual's addition (include/norm.h), forward and backward; its first half for the norm in
// front of a W8A8 Linear layer (include/w8a8.h), whose second half is the quantisation (k_w8a8.hip).
//
// A team of T threads per row: a wavefront up to 2048 features, a workgroup of 256 to 512 up to 8192, of 1024 up to 16384.  The row stays
// in registers between the sum of its squares and its result, so every tensor is read or written once: bound by HBM.
#include "rows.h"

namespace sla {

template <bool NT = false>
__device__ __forceinline__ uint4 load_row(const bf16_t* row, int e) { return load_from<NT, uint4>(row + 8ll * e); }

// STATS: h and r instead of h and y.
template <int T, int CH, bool STATS, bool NT>
__global__ void __launch_bounds__(T == 64 ? 256 : T) norm_fwd_kernel(const bf16_t* __restrict__ x, const bf16_t* __restrict__ res,
                                                                         const bf16_t* __restrict__ weight, bf16_t* __restrict__ h,
                                                                         bf16_t* __restrict__ y, float* __restrict__ r_out, int M, int K,
                                                                         float eps) {
  __shared__ float red[2][T / 64];
  constexpr int TEAMS = T == 64 ? 4 : 1;
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x, n = K / 8;
  int turn = 0;
  for (long long m = (long long)TEAMS * blockIdx.x + (T == 64 ? threadIdx.x >> 6 : 0); m < M; m += (long long)TEAMS * gridDim.x, turn ^= 1) {
    uint4 v[CH], add[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      v[c] = add[c] = uint4{0u, 0u, 0u, 0u};
      if (t + c * T < n) {
        v[c] = load_row<NT>(x + m * K, t + c * T);
        if (res) add[c] = load_row<NT>(res + m * K, t + c * T);
      }
    }
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float a[8];
      unpack8(v[c], a);
      if (res) {
        float b[8];
        unpack8(add[c], b);
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] += b[i];
        v[c] = pack8(a);
        if (t + c * T < n) store_to<NT && !STATS>(h + m * K + 8ll * (t + c * T), v[c]);   // (STATS: h is read again at once)
        unpack8(v[c], a);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(a[i], a[i], ss);
    }
    const float r = __builtin_amdgcn_rsqf(team_sum<T>(ss, red[turn]) / (float)K + eps);
    if constexpr (STATS) {
      if (t == 0) r_out[m] = r;
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if (t + c * T >= n) break;
        float a[8];
        unpack8(v[c], a);
        if (weight) {
          float w[8];
          unpack8(load_row(weight, t + c * T), w);
#pragma unroll
          for (int i = 0; i < 8; ++i) a[i] = a[i] * r * w[i];
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) a[i] *= r;
        }
        store_to<NT>(y + m * K + 8ll * (t + c * T), pack8(a));
      }
    }
  }
}

// dx, and each workgroup's share of dw in registers over the rows it takes.
template <int T, int CH, bool NT>
__global__ void __launch_bounds__(T == 64 ? 256 : T) norm_bwd_kernel(const bf16_t* __restrict__ dy, const bf16_t* __restrict__ dh,
                                                                         const bf16_t* __restrict__ h, const bf16_t* __restrict__ weight,
                                                                         bf16_t* __restrict__ dx, float* __restrict__ part, int M, int K,
                                                                         float eps) {
  __shared__ float red[2][2][T / 64];
  __shared__ float4 join[T == 64 ? 2 * CH * 64 : 1];
  constexpr int TEAMS = T == 64 ? 4 : 1;
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x, wave = threadIdx.x >> 6, n = K / 8;
  const float inv = 1.0f / (float)K;
  float dw[CH][8] = {};
  int turn = 0;
  for (long long m = (long long)TEAMS * blockIdx.x + (T == 64 ? wave : 0); m < M; m += (long long)TEAMS * gridDim.x, turn ^= 1) {
    uint4 rg[CH], rx[CH], rh[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      rg[c] = rx[c] = rh[c] = uint4{0u, 0u, 0u, 0u};
      if (t + c * T < n) {
        rg[c] = load_row<NT>(dy + m * K, t + c * T);
        rx[c] = load_row<NT>(h + m * K, t + c * T);
        if (dh) rh[c] = load_row<NT>(dh + m * K, t + c * T);
      }
    }
    // of one share: h, w dy, and dy h (the share of dw is r times that)
    auto share = [&](int c, float (&x)[8], float (&g)[8], float (&gx)[8]) __attribute__((always_inline)) {
      unpack8(rx[c], x);
      unpack8(rg[c], g);
#pragma unroll
      for (int i = 0; i < 8; ++i) gx[i] = g[i] * x[i];
      if (weight) {
        float w[8];
        unpack8(load_row(weight, min(t + c * T, n - 1)), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] *= w[i];
      }
    };
    float ss = 0.f, xg = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float x[8], g[8], gx[8];
      share(c, x, g, gx);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ss = __builtin_fmaf(x[i], x[i], ss);
        xg = __builtin_fmaf(x[i], g[i], xg);
      }
    }
    ss = rows_sum(row_sum(ss));
    xg = rows_sum(row_sum(xg));
    if constexpr (T > 64) {
      if ((threadIdx.x & 63) == 0) { red[turn][0][wave] = ss; red[turn][1][wave] = xg; }
      __syncthreads();
      ss = xg = 0.f;
#pragma unroll
      for (int i = 0; i < T / 64; ++i) { ss += red[turn][0][i]; xg += red[turn][1][i]; }
    }
    // (dx = r (g - x r^2 mean(x g)): r^3 need not be a number of fp32, r is up to 1 / sqrt(eps))
    const float r = __builtin_amdgcn_rsqf(ss * inv + eps), dot = xg * inv * r * r;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float x[8], g[8], gx[8], up[8];
      share(c, x, g, gx);
      unpack8(rh[c], up);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dw[c][i] = __builtin_fmaf(gx[i], r, dw[c][i]);
        up[i] = __builtin_fmaf(__builtin_fmaf(-x[i], dot, g[i]), r, up[i]);
      }
      if (t + c * T < n) store_to<NT>(dx + m * K + 8ll * (t + c * T), pack8(up));
    }
  }
  if (!part) return;
  auto f4 = [](const float* a) __attribute__((always_inline)) { return float4{a[0], a[1], a[2], a[3]}; };
  float* mine = part + (long long)blockIdx.x * K;
  if constexpr (T == 64) {                     // four wavefronts hold shares of the same features
    for (int k = 0; k < 4; ++k) {
      if (wave == k) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float4 s = f4(dw[c] + 4 * u);
            if (k > 0) {
              const float4 p = join[(2 * c + u) * 64 + t];
              s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
            }
            join[(2 * c + u) * 64 + t] = s;
          }
      }
      __syncthreads();
    }
    if (wave == 0) {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (t + c * T < n) {
          *(float4*)(mine + 8 * (t + c * T)) = join[2 * c * 64 + t];
          *(float4*)(mine + 8 * (t + c * T) + 4) = join[(2 * c + 1) * 64 + t];
        }
    }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (t + c * T < n) {
        *(float4*)(mine + 8 * (t + c * T)) = f4(dw[c]);
        *(float4*)(mine + 8 * (t + c * T) + 4) = f4(dw[c] + 4);
      }
  }
}

// ---------------------------------------------------------------------------
// The team and the shares of a thread for K features: F(T, CH).  In the forward direction, from 2056 to 8192 features, threads are fitted
// to two shares each, in steps of at most a third; beyond, 1024 threads take whatever there is.  With 256 threads of three for 5120
// features, a sixth of them idle, 75600 rows took 529 us, now 518; 6144 160 / 156.  The gradient, whose threads hold sums of dw too,
// takes three of 256 threads there (568 us; with 320 586; 6144 184 / 207), but two of 512 for 8192 (265 / 231).
#define NORM_TEAMS(K, F)                  \
  do {                                    \
    const int n_ = (K) / 8;               \
    if (n_ <= 64) F(64, 1);               \
    else if (n_ <= 128) F(64, 2);         \
    else if (n_ <= 192) F(64, 3);         \
    else if (n_ <= 256) F(64, 4);         \
    else if (n_ <= 512) F(256, 2);        \
    else if (n_ <= 640) F(320, 2);        \
    else if (n_ <= 768) F(384, 2);        \
    else if (n_ <= 1024) F(512, 2);       \
    else F(1024, 2);                      \
  } while (0)
#define NORM_BWD_TEAMS(K, F)              \
  do {                                    \
    const int n_ = (K) / 8;               \
    if (n_ <= 64) F(64, 1);               \
    else if (n_ <= 128) F(64, 2);         \
    else if (n_ <= 192) F(64, 3);         \
    else if (n_ <= 256) F(64, 4);         \
    else if (n_ <= 512) F(256, 2);        \
    else if (n_ <= 768) F(256, 3);        \
    else if (n_ <= 1024) F(512, 2);       \
    else F(1024, 2);                      \
  } while (0)

// `tensors` of these that do not fit the memory-side cache together are read and written past it.
static bool streams(int M, int K, int tensors) { return (long long)M * K * 2 * tensors > (256ll << 20); }
static unsigned row_workgroups(int M, int T) { return (unsigned)min(T == 64 ? (M + 3) / 4 : M, 1 << 20); }

void launch_norm_fwd(const void* x, const void* res, const void* w, void* h, void* y, int M, int K, float eps, hipStream_t stream) {
#define NORM_FWD(T, CH)                                                                                                   \
  do {                                                                                                                    \
    if (streams(M, K, res ? 4 : 2)) NORM_FWD_(T, CH, true); else NORM_FWD_(T, CH, false);                                 \
  } while (0)
#define NORM_FWD_(T, CH, NT)                                                                                              \
  norm_fwd_kernel<T, CH, false, NT><<<row_workgroups(M, T), T == 64 ? 256 : T, 0, stream>>>(                         \
      (const bf16_t*)x, (const bf16_t*)res, (const bf16_t*)w, (bf16_t*)h, (bf16_t*)y, nullptr, M, K, eps)
  NORM_TEAMS(K, NORM_FWD);
#undef NORM_FWD_
#undef NORM_FWD
}
void launch_norm_stats(const void* x, const void* res, void* h, float* r, int M, int K, float eps, hipStream_t stream) {
#define NORM_STATS(T, CH)                                                                                                 \
  do {                                                                                                                    \
    if (res && streams(M, K, 3)) NORM_STATS_(T, CH, true); else NORM_STATS_(T, CH, false);                                \
  } while (0)
#define NORM_STATS_(T, CH, NT)                                                                                            \
  norm_fwd_kernel<T, CH, true, NT><<<row_workgroups(M, T), T == 64 ? 256 : T, 0, stream>>>(                          \
      (const bf16_t*)x, (const bf16_t*)res, nullptr, (bf16_t*)h, nullptr, r, M, K, eps)
  NORM_TEAMS(K, NORM_STATS);
#undef NORM_STATS_
#undef NORM_STATS
}

// Each workgroup leaves a row of partial sums of dw: at least eight rows (of each team) for one of those, but enough workgroups to
// fill the chip.  In us, with 256 / 512 / 1024 workgroups: 2048 x 5120 28.2 / 26.2 / 29.0, 4096 x 5120 45.5 / 38.9 / 39.6, 8192 x 5120
// 96.2 / 79.3 / 75.2, 8192 x 1536 29.3 / 26.4 / 27.8; of 1024 threads, 2048 x 13824 46.3 / 53.1 / 68.8, 8192 x 13824 with 512 181.
int norm_bwd_workgroups(int M, int K) {
  const int all = K <= 2048 ? (M + 3) / 4 : M, least = K <= 8192 ? 512 : 256;
  return min(all, max(least, min(all / 8, 2 * least)));
}
void launch_norm_bwd(const void* dy, const void* dh, const void* h, const void* w, void* dx, float* dw, float* part, int M, int K,
                     float eps, hipStream_t stream) {
  if (!dw) part = nullptr;
  const unsigned grid = (unsigned)norm_bwd_workgroups(M, K);
#define NORM_BWD(T, CH)                                                                                                   \
  do {                                                                                                                    \
    if (streams(M, K, dh ? 4 : 3)) NORM_BWD_(T, CH, true); else NORM_BWD_(T, CH, false);                                  \
  } while (0)
#define NORM_BWD_(T, CH, NT)                                                                                              \
  norm_bwd_kernel<T, CH, NT><<<grid, T == 64 ? 256 : T, 0, stream>>>((const bf16_t*)dy, (const bf16_t*)dh, (const bf16_t*)h, \
                                                                         (const bf16_t*)w, (bf16_t*)dx, part, M, K, eps)
  NORM_BWD_TEAMS(K, NORM_BWD);
#undef NORM_BWD_
#undef NORM_BWD
  PartialSums s{};
  s.part[0] = part;
  s.dw[0] = dw;
  s.width[0] = K;
  s.n_part = (int)grid;
  launch_sum_partials(s, stream);
}

}  // namespace sla
