// Layer norm with gate and modulation (include/norm.h), forward and backward; the forward pass into the codes of a 4-bit layer
// (include/mxfp4.h) as well.
//
// A team of T threads per row, as in k_norm.hip: the row stays in registers between its sums and its result, so every tensor
// is read or written once: bound by HBM.  Mean first, then the sum of the squared deviations from it.
#include "layer.h"
#include "mxfp4.h"

namespace sla {

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// MX: codes instead of y.
template <int T, int CH, bool MX, bool NT>
__global__ void __launch_bounds__(T == 64 ? 256 : T) layer_fwd_kernel(LayerArgs a) {
  __shared__ float red[2][T / 64];
  constexpr int TEAMS = T == 64 ? 4 : 1;
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x, n = a.K / 8;
  const long long K = a.K;
  const float inv = 1.0f / (float)a.K;
  for (long long m = (long long)TEAMS * blockIdx.x + (T == 64 ? threadIdx.x >> 6 : 0); m < a.M; m += (long long)TEAMS * gridDim.x) {
    const long long s = (int)m / a.rows;
    uint4 v[CH], add[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      v[c] = add[c] = uint4{0u, 0u, 0u, 0u};
      if (t + c * T < n) {
        v[c] = load_from<NT, uint4>(a.x + m * K + 8ll * (t + c * T));
        if (a.res) add[c] = load_from<NT, uint4>(a.res + m * K + 8ll * (t + c * T));
      }
    }
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float x[8];
      unpack8(v[c], x);
      if (a.res && t + c * T < n) {
        float r[8];
        unpack8(add[c], r);
        if (a.gate.v) {
          float g[8];
          load8(a.gate.v + s * a.gate.stride + 8 * (t + c * T), g);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(g[i], r[i], x[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] += r[i];
        }
        v[c] = pack8(x);
        store_to<NT>(a.h + m * K + 8ll * (t + c * T), v[c]);
        unpack8(v[c], x);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i];
    }
    const float mean = team_sum<T>(sum, red[0]) * inv;
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (t + c * T >= n) break;
      float x[8];
      unpack8(v[c], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i] - mean, x[i] - mean, ss);
    }
    const float r = __builtin_amdgcn_rsqf(team_sum<T>(ss, red[1]) * inv + a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int e = t + c * T;
      uint4 out = uint4{0u, 0u, 0u, 0u};
      if (e < n) {
        float x[8], u[8];
        unpack8(v[c], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (x[i] - mean) * r;
        if (a.w) {
          unpack8(*(const uint4*)(a.w + 8 * e), u);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= u[i];
        }
        if (a.b) {
          unpack8(*(const uint4*)(a.b + 8 * e), u);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] += u[i];
        }
        if (a.scale.v) {
          load8(a.scale.v + s * a.scale.stride + 8 * e, u);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(x[i], u[i], x[i]);
        }
        if (a.shift.v) {
          load8(a.shift.v + s * a.shift.stride + 8 * e, u);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] += u[i];
        }
        out = pack8(x);
      }
      if constexpr (MX) {
        if (e < mx_steps(a.K) * (MX_STEP / 8)) mx_store8(out, (int)m, e, mx_rows(a.M), a.codes, a.exps);
      } else {
        if (e < n) store_to<NT>(a.y + m * K + 8ll * e, out);
      }
    }
  }
}

// dx, dres, and each workgroup's shares of the sums over a sample's rows: S0 of dy, S1 of dy o n, S2 of dx o res, each
// [workgroups, K].  Workgroup s * chunks + j takes rows j * per .. of sample s.
template <int T, int CH, bool GATE, bool NT>
__global__ void __launch_bounds__(T == 64 ? 256 : T) layer_bwd_kernel(LayerBwdArgs a, int chunks, int per, float* s0, float* s1,
                                                                       float* s2) {
  __shared__ float red[T / 64], red3[3][T / 64];
  __shared__ float4 join[T == 64 ? 6 * CH * 64 : 1];
  constexpr int TEAMS = T == 64 ? 4 : 1;
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x, wave = threadIdx.x >> 6, n = a.K / 8;
  const long long K = a.K;
  const float inv = 1.0f / (float)a.K;
  const int s = blockIdx.x / chunks, j = blockIdx.x - s * chunks;
  const long long first = (long long)s * a.rows + (long long)j * per;
  const long long last = min((long long)a.M, min((long long)(s + 1) * a.rows, first + per));
  float a0[CH][8] = {}, a1[CH][8] = {}, a2[GATE ? CH : 1][8] = {};
  for (long long m = first + (T == 64 ? wave : 0); m < last; m += TEAMS) {
    // The vectors are the same in every row: they stay in registers, 20 a share, but where a thread has four shares (`again` hides
    // that they are; and res is then read where it is needed).
    int again = 0;
    if constexpr (CH > 3) asm volatile("" : "+s"(again));
    uint4 rg[CH], rx[CH], rh[CH], rr[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      rg[c] = rx[c] = rh[c] = rr[c] = uint4{0u, 0u, 0u, 0u};
      if (t + c * T < n) {
        rg[c] = load_from<NT, uint4>(a.dy + m * K + 8ll * (t + c * T));
        rx[c] = load_from<NT, uint4>(a.h + m * K + 8ll * (t + c * T));
        if (a.dh) rh[c] = load_from<NT, uint4>(a.dh + m * K + 8ll * (t + c * T));
        if (GATE && CH <= 3 && a.res) rr[c] = load_from<NT, uint4>(a.res + m * K + 8ll * (t + c * T));
      }
    }
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float x[8];
      unpack8(rx[c], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i];
    }
    const float mean = team_sum<T>(sum, red) * inv;
    // of one share: h - mean and g = dy o (1 + scale) o w, both zero where there are no features
    auto share = [&](int c, float (&x)[8], float (&g)[8]) __attribute__((always_inline)) {
      const int e = min(t + c * T, n - 1) + again;
      unpack8(rx[c], x);
      unpack8(rg[c], g);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = t + c * T < n ? x[i] - mean : 0.f;
      float u[8];
      if (a.scale.v) {
        load8(a.scale.v + s * a.scale.stride + 8 * e, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = __builtin_fmaf(g[i], u[i], g[i]);
      }
      if (a.w) {
        unpack8(*(const uint4*)(a.w + 8 * e), u);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] *= u[i];
      }
    };
    float ss = 0.f, sg = 0.f, xg = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float x[8], g[8];
      share(c, x, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ss = __builtin_fmaf(x[i], x[i], ss);
        sg += g[i];
        xg = __builtin_fmaf(x[i], g[i], xg);
      }
    }
    ss = rows_sum(row_sum(ss));
    sg = rows_sum(row_sum(sg));
    xg = rows_sum(row_sum(xg));
    if constexpr (T > 64) {
      if ((threadIdx.x & 63) == 0) { red3[0][wave] = ss; red3[1][wave] = sg; red3[2][wave] = xg; }
      __syncthreads();
      ss = sg = xg = 0.f;
#pragma unroll
      for (int i = 0; i < T / 64; ++i) { ss += red3[0][i]; sg += red3[1][i]; xg += red3[2][i]; }
    }
    // (dx = dh + r (g - mean(g) - x r^2 mean(x g)): r^2 mean(x g) as two products, r is up to 1 / sqrt(eps))
    const float r = __builtin_amdgcn_rsqf(ss * inv + a.eps), dot = xg * inv * r * r, mg = sg * inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int e = t + c * T;
      float x[8], g[8], d[8], u[8];
      if (GATE && CH > 3 && a.res && e < n) rr[c] = load_from<NT, uint4>(a.res + m * K + 8ll * e);
      share(c, x, g);
      unpack8(rg[c], u);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a0[c][i] += u[i];
        a1[c][i] = __builtin_fmaf(u[i], x[i] * r, a1[c][i]);
      }
      unpack8(rh[c], d);
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = __builtin_fmaf(__builtin_fmaf(-x[i], dot, g[i] - mg), r, d[i]);
      if (e < n) store_to<NT>(a.dx + m * K + 8ll * e, pack8(d));
      if constexpr (GATE) {
        unpack8(rr[c], u);
#pragma unroll
        for (int i = 0; i < 8; ++i) a2[c][i] = __builtin_fmaf(d[i], u[i], a2[c][i]);
        if (a.dres && e < n) {
          load8(a.gate.v + s * a.gate.stride + 8 * (e + again), u);
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] *= u[i];
          store_to<NT>(a.dres + m * K + 8ll * e, pack8(d));
        }
      }
      if constexpr (CH > 3) __builtin_amdgcn_sched_barrier(0);
    }
  }
  auto f4 = [](const float* x) __attribute__((always_inline)) { return float4{x[0], x[1], x[2], x[3]}; };
  auto leave = [&](float* to, const float (&acc)[CH][8], float4* mine) __attribute__((always_inline)) {
    if (!to) return;
    to += (long long)blockIdx.x * K;
    if constexpr (T == 64) {                   // four wavefronts hold shares of the same features
      for (int k = 0; k < 4; ++k) {
        if (wave == k) {
#pragma unroll
          for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              float4 v = f4(acc[c] + 4 * u);
              if (k > 0) {
                const float4 p = mine[(2 * c + u) * 64 + t];
                v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
              }
              mine[(2 * c + u) * 64 + t] = v;
            }
        }
        __syncthreads();
      }
      if (wave == 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
          if (t + c * T < n) {
            *(float4*)(to + 8 * (t + c * T)) = mine[2 * c * 64 + t];
            *(float4*)(to + 8 * (t + c * T) + 4) = mine[(2 * c + 1) * 64 + t];
          }
      }
    } else {
#pragma unroll
      for (int c = 0; c < CH; ++c)
        if (t + c * T < n) {
          *(float4*)(to + 8 * (t + c * T)) = f4(acc[c]);
          *(float4*)(to + 8 * (t + c * T) + 4) = f4(acc[c] + 4);
        }
    }
  };
  leave(s0, a0, join);
  leave(s1, a1, join + (T == 64 ? 2 * CH * 64 : 0));
  if constexpr (GATE) leave(s2, a2, join + (T == 64 ? 4 * CH * 64 : 0));
}

// A sample's sums from its workgroups' shares, in a fixed order, and the gradients they give: workgroup (sample, 64 columns),
// 16 threads of four adjacent columns, 16 along the shares.  With several samples, what each adds to dw and db goes to
// pw, pb [samples, K], which launch_sum_partials adds up.
constexpr int LSUM_ENTRIES = 64;
__global__ void __launch_bounds__(256) layer_sums_kernel(LayerBwdArgs a, int chunks, const float* s0, const float* s1,
                                                         const float* s2, float* pw, float* pb) {
  __shared__ float4 red[3][16][16];
  const int blocks = (a.K + LSUM_ENTRIES - 1) / LSUM_ENTRIES, s = blockIdx.x / blocks;
  const int t = threadIdx.x, col = t & 15, row = t >> 4, x = (blockIdx.x - s * blocks) * LSUM_ENTRIES + 4 * col;
  auto add = [](float4& a, const float4& b) __attribute__((always_inline)) { a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; };
  const float* src[3] = {s0, s1, s2};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    float4 v[4] = {};
    if (src[k] && x < a.K) {
      const float* part = src[k] + (long long)s * chunks * a.K + x;
      int p = row;
      for (; p + 48 < chunks; p += 64)
#pragma unroll
        for (int u = 0; u < 4; ++u) add(v[u], *(const float4*)(part + (long long)(p + 16 * u) * a.K));
      for (; p < chunks; p += 16) add(v[0], *(const float4*)(part + (long long)p * a.K));
    }
    add(v[0], v[1]);
    add(v[2], v[3]);
    add(v[0], v[2]);
    red[k][row][col] = v[0];
  }
  __syncthreads();
  if (t >= 16 || x >= a.K) return;
  float4 sum[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    float4 r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = red[k][i][t];
#pragma unroll
    for (int step = 1; step < 16; step *= 2)
#pragma unroll
      for (int i = 0; i < 16; i += 2 * step) add(r[i], r[i + step]);
    sum[k] = r[0];
  }
  const long long at = (long long)s * a.K + x;
  const float v0[4] = {sum[0].x, sum[0].y, sum[0].z, sum[0].w}, v1[4] = {sum[1].x, sum[1].y, sum[1].z, sum[1].w};
  float up[4] = {1.f, 1.f, 1.f, 1.f}, w[4] = {1.f, 1.f, 1.f, 1.f}, b[4] = {}, ds[4], dw[4], db[4];
  if (a.scale.v) {
    const float4 u = *(const float4*)(a.scale.v + s * a.scale.stride + x);
    up[0] += u.x; up[1] += u.y; up[2] += u.z; up[3] += u.w;
  }
  auto four = [&](const bf16_t* p, float (&v)[4]) __attribute__((always_inline)) {
    const uint2 q = *(const uint2*)(p + x);
    v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
  };
  if (a.w) four(a.w, w);
  if (a.b) four(a.b, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    ds[i] = __builtin_fmaf(w[i], v1[i], b[i] * v0[i]);
    dw[i] = up[i] * v1[i];
    db[i] = up[i] * v0[i];
  }
  if (a.grads.shift) *(float4*)(a.grads.shift + at) = sum[0];
  if (a.grads.scale) *(float4*)(a.grads.scale + at) = float4{ds[0], ds[1], ds[2], ds[3]};
  if (a.grads.gate) *(float4*)(a.grads.gate + at) = sum[2];
  if (pw) *(float4*)(pw + at) = float4{dw[0], dw[1], dw[2], dw[3]};
  if (pb) *(float4*)(pb + at) = float4{db[0], db[1], db[2], db[3]};
}

// ---------------------------------------------------------------------------
// The team and the shares of a thread for n shares of eight features: F(T, CH).
#define LAYER_TEAMS(n, F)                 \
  do {                                    \
    const int n_ = (n);                   \
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
#define LAYER_BWD_TEAMS(n, F)             \
  do {                                    \
    const int n_ = (n);                   \
    if (n_ <= 64) F(64, 1);               \
    else if (n_ <= 128) F(64, 2);         \
    else if (n_ <= 192) F(64, 3);         \
    else if (n_ <= 256) F(64, 4);         \
    else if (n_ <= 512) F(256, 2);        \
    else if (n_ <= 768) F(256, 3);        \
    else if (n_ <= 1024) F(512, 2);       \
    else F(512, 4);                       \
  } while (0)

// `tensors` of these that do not fit the memory-side cache together are read and written past it.
static bool streams(int M, int K, int tensors) { return (long long)M * K * 2 * tensors > (256ll << 20); }

void launch_layer_fwd(const LayerArgs& a, hipStream_t stream) {
  const bool nt = streams(a.M, a.K, a.res ? 4 : 2);
#define LAYER_FWD(T, CH)                                                                  \
  do {                                                                                    \
    const unsigned grid = (unsigned)min(T == 64 ? (a.M + 3) / 4 : a.M, 1 << 20);          \
    constexpr int threads = T == 64 ? 256 : T;                                            \
    if (a.codes) {                                                                        \
      if (nt) layer_fwd_kernel<T, CH, true, true><<<grid, threads, 0, stream>>>(a);       \
      else layer_fwd_kernel<T, CH, true, false><<<grid, threads, 0, stream>>>(a);         \
    } else {                                                                              \
      if (nt) layer_fwd_kernel<T, CH, false, true><<<grid, threads, 0, stream>>>(a);      \
      else layer_fwd_kernel<T, CH, false, false><<<grid, threads, 0, stream>>>(a);        \
    }                                                                                     \
  } while (0)
  LAYER_TEAMS(a.codes ? mx_steps(a.K) * (MX_STEP / 8) : a.K / 8, LAYER_FWD);   // (codes: those behind the last feature too)
#undef LAYER_FWD
}

// How a sample's rows are dealt: at least eight to a workgroup (to a team), but enough workgroups to fill the chip.
struct LayerDeal { int samples, chunks, per; };
static LayerDeal layer_deal(int M, int K, int rows) {
  rows = min(rows, M);
  const int samples = (M + rows - 1) / rows, teams = K <= 2048 ? 4 : 1, most = K <= 8192 ? 1024 : 512;
  const int all = (rows + teams - 1) / teams;                              // chunks of one row per team
  const int want = max(1, (min(most, max(most / 2, M / (8 * teams))) + samples - 1) / samples);
  const int per = teams * ((all + min(all, want) - 1) / min(all, want));
  return {samples, (rows + per - 1) / per, per};
}
// three sums per workgroup, and each sample's share of dw and db
size_t layer_bwd_bytes(int M, int K, int rows) {
  const LayerDeal d = layer_deal(M, K, rows);
  return 3 * align256((size_t)d.samples * d.chunks * K * 4) + (d.samples > 1 ? 2 * align256((size_t)d.samples * K * 4) : 0);
}

void launch_layer_bwd(const LayerBwdArgs& a, hipStream_t stream) {
  const LayerDeal d = layer_deal(a.M, a.K, a.rows);
  const norm_layer_grads& g = a.grads;
  const size_t one = align256((size_t)d.samples * d.chunks * a.K * 4), per_sample = align256((size_t)d.samples * a.K * 4);
  unsigned char* ws = (unsigned char*)a.ws;
  const bool sums = g.w || g.b || g.scale || g.shift;
  float *s0 = sums ? (float*)ws : nullptr, *s1 = sums ? (float*)(ws + one) : nullptr, *s2 = g.gate ? (float*)(ws + 2 * one) : nullptr;
  const unsigned grid = (unsigned)d.samples * d.chunks;
  const bool gate = a.gate.v != nullptr, nt = streams(a.M, a.K, 3 + (a.dh != nullptr) + 2 * gate);
#define LAYER_BWD(T, CH)                                                                                            \
  do {                                                                                                              \
    constexpr int threads = T == 64 ? 256 : T;                                                                      \
    if (gate) {                                                                                                     \
      if (nt) layer_bwd_kernel<T, CH, true, true><<<grid, threads, 0, stream>>>(a, d.chunks, d.per, s0, s1, s2);    \
      else layer_bwd_kernel<T, CH, true, false><<<grid, threads, 0, stream>>>(a, d.chunks, d.per, s0, s1, s2);      \
    } else {                                                                                                        \
      if (nt) layer_bwd_kernel<T, CH, false, true><<<grid, threads, 0, stream>>>(a, d.chunks, d.per, s0, s1, s2);   \
      else layer_bwd_kernel<T, CH, false, false><<<grid, threads, 0, stream>>>(a, d.chunks, d.per, s0, s1, s2);     \
    }                                                                                                               \
  } while (0)
  LAYER_BWD_TEAMS(a.K / 8, LAYER_BWD);
#undef LAYER_BWD
  if (!sums && !g.gate) return;
  float *pw = g.w, *pb = g.b;
  if (d.samples > 1) {
    pw = g.w ? (float*)(ws + 3 * one) : nullptr;
    pb = g.b ? (float*)(ws + 3 * one + per_sample) : nullptr;
  }
  layer_sums_kernel<<<(unsigned)d.samples * ((a.K + LSUM_ENTRIES - 1) / LSUM_ENTRIES), 256, 0, stream>>>(a, d.chunks, s0, s1, s2, pw, pb);
  if (d.samples > 1 && (g.w || g.b)) {
    PartialSums p{};
    p.part[0] = pw; p.dw[0] = g.w; p.width[0] = a.K;
    p.part[1] = pb; p.dw[1] = g.b; p.width[1] = a.K;
    p.n_part = d.samples;
    launch_sum_partials(p, stream);
  }
}

}  // namespace sla
