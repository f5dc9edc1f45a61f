// Layer norm with gate and modulation (include/norm.h), forward and backward; the forward pass into the codes of a 4-bit layer
// (include/mxfp4.h) as well.
//
// A team of T threads per row, as in k_norm.hip: the row stays in registers between its sums and its result, so every tensor
// is read or written once: bound by HBM (a copy reaches 4.9 TB/s, an addition of two tensors 5.8).  All in fp32; the stored stream is rounded to
// bf16 before it is normed, because its readers find it so, the result once.
// Two passes over registers: the sum S of the row, of which row_mean makes p, the bf16 number next to the mean, and c = (S - K p) / K, the rest of
// it; then the sum of (x - p)^2.  The deviations are (x - p) - c, the variance mean((x - p)^2) - c^2.  So the rounding of the mean is in no
// deviation (deviations from the rounded mean put 0.7 % on the n of 999 equal features beside one that is a bf16 step larger, and the n of
// constant rows up to 1): differences of bf16 numbers are exact, or off by 2^-24 of themselves, and those of a constant row zero, c too.  S is
// exact in fp32 where a row's features are within a factor of four (at most 2^14 numbers of 10 bits), and else its rounding is small against the
// deviations (n off by 2^-18 at most in 2400 rows with features of any other size among equal ones).  Nor do the squares cancel: no x lies
// between the bf16 numbers a < b around the mean, so (x - a)(x - b) >= 0 and the variance is at least (mean - a)(b - mean), which is at least
// c^2, p being the nearer of the two.
// Measured: forward with gate and modulation 75600 x 5120 537 us, 5.8 TB/s, 32760 x 5120 230 (5.8), 65520 x 1536 138 (5.8), 20000 x 13824 397, x
// alone 75600 x 5120 243 (6.4); into codes 75600 x 5120 460 (5.5), 65520 x 1536 121; one row of 5120 2.9.  Backward with everything
// 65520 x 1536 253 us, 4.8 TB/s, 32760 x 5120 402 (5.0), 8192 x 5120 123, 129 x 1536 12.
#include "layer.h"
#include "mxfp4.h"

namespace sla {

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// Share e of a row: its address is the row's, the same for a wavefront, and 32 bits of each lane's.
__device__ __forceinline__ const bf16_t* share_of(const bf16_t* row, int e) { return (const bf16_t*)((const char*)row + 16u * (unsigned)e); }
__device__ __forceinline__ bf16_t* share_of(bf16_t* row, int e) { return (bf16_t*)((char*)row + 16u * (unsigned)e); }

// p and c of a row whose K features have the sum s.
struct RowMean { float p, c; };
__device__ __forceinline__ RowMean row_mean(float s, float K, float inv) {
  const float p = bf16_lo(pack_bf16x2(s * inv, 0.f));
  return {p, __builtin_fmaf(-K, p, s) * inv};
}
// 1 / sqrt(variance + eps), given mean((x - p)^2) and c.  (Rounded, the variance could fall below zero.)
__device__ __forceinline__ float row_factor(float square, float c, float eps) {
  return __builtin_amdgcn_rsqf(__builtin_fmaxf(__builtin_fmaf(-c, c, square), 0.f) + eps);
}

// MX: codes instead of y.  A team takes ROWS rows of one sample at a time: two share what they read of the vectors, which come from the
// caches, 12 bytes a feature with a gate, scale and shift.
template <int T, int CH, int ROWS, bool MX, bool NT>
__global__ void __launch_bounds__(T == 64 ? 256 : T) layer_fwd_kernel(LayerArgs a, int groups, int per_sample) {
  __shared__ float red[2][ROWS][T / 64];
  constexpr int TEAMS = T == 64 ? 4 : 1;
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = a.K / 8;
  int block = blockIdx.x, blocks = gridDim.x;
  if constexpr (T == 1024) {                   // (of a grid of two rows, see launch_layer_fwd)
    block += blockIdx.y * blocks;
    blocks *= gridDim.y;
  }
  if constexpr (MX) {
    // Workgroups are dealt round-robin over the 8 XCDs: of every 8 RUN, RUN neighbours to each, so that the 16 rows whose exponents
    // share a line are one L2's.
    constexpr int RUN = 16 / (ROWS * TEAMS);
    const int from = block / (8 * RUN) * (8 * RUN);
    if (from + 8 * RUN <= blocks) block = from + ((block - from) & 7) * RUN + ((block - from) >> 3);
  }
  const int group = TEAMS * block + (T == 64 ? wave : 0);
  if (group >= groups) return;                 // (T > 64: the whole workgroup)
  const long long K = a.K;
  const float inv = 1.0f / (float)a.K;
  const int s = group / per_sample;
  const long long m = (long long)s * a.rows + (long long)ROWS * (group - s * per_sample);
  // (a second row that is not there: the first once more, nothing of it is stored)
  const bool second = ROWS == 2 && m + 1 < a.M && m + 1 < (long long)(s + 1) * a.rows;
  auto there = [&](int r) { return r == 0 || second; };
  auto row = [&](int r) { return m + (there(r) ? r : 0); };
  // sums of one number per row over the team
  auto sums = [&](float (&x)[ROWS], float (*mem)[T / 64]) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) x[r] = rows_sum(row_sum(x[r]));
    if constexpr (T > 64) {
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) mem[r][wave] = x[r];
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        x[r] = 0.f;
#pragma unroll
        for (int i = 0; i < T / 64; ++i) x[r] += mem[r][i];
      }
    }
  };
  uint4 v[ROWS][CH], add[ROWS][CH];
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      v[r][c] = add[r][c] = uint4{0u, 0u, 0u, 0u};
      if (t + c * T < n) {
        v[r][c] = load_from<NT, uint4>(share_of(a.x + row(r) * K, t + c * T));
        if (a.res) add[r][c] = load_from<NT, uint4>(share_of(a.res + row(r) * K, t + c * T));
      }
    }
  // The vectors: of a lone wavefront requested before they are needed, behind what is waited for first, the rows and the sums (65520 x 1536
  // 153 -> 141 us); of a workgroup when they are needed, there it is the registers that count (75600 x 5120 561 -> 541).
  constexpr bool EARLY = T == 64;
  float g[CH][8], sc[CH][8], sh[CH][8];
  uint4 w[CH] = {}, b[CH] = {};
  auto gate = [&](int c) __attribute__((always_inline)) {
    if (a.gate.v) load8(a.gate.v + s * a.gate.stride + 8 * min(t + c * T, n - 1), g[c]);
  };
  auto vectors = [&](int c) __attribute__((always_inline)) {
    const int e = min(t + c * T, n - 1);
    if (a.w) w[c] = *(const uint4*)(a.w + 8 * e);
    if (a.b) b[c] = *(const uint4*)(a.b + 8 * e);
    if (a.scale.v) load8(a.scale.v + s * a.scale.stride + 8 * e, sc[c]);
    if (a.shift.v) load8(a.shift.v + s * a.shift.stride + 8 * e, sh[c]);
  };
  if constexpr (EARLY) {
#pragma unroll
    for (int c = 0; c < CH; ++c) gate(c);
  }
  float sum[ROWS] = {}, rs[ROWS] = {};
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int e = t + c * T;
    if (e >= n) break;
    if constexpr (!EARLY) gate(c);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float x[8], u[8];
      unpack8(v[r][c], x);
      if (a.res) {
        unpack8(add[r][c], u);
        if (a.gate.v) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(g[c][i], u[i], x[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] += u[i];
        }
        v[r][c] = pack8(x);
        if (there(r)) store_to<NT>(share_of(a.h + row(r) * K, e), v[r][c]);
        unpack8(v[r][c], x);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[r] += x[i];
    }
  }
  if constexpr (EARLY) {
#pragma unroll
    for (int c = 0; c < CH; ++c) vectors(c);
  }
  sums(sum, red[0]);
  RowMean mean[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    mean[r] = row_mean(sum[r], (float)a.K, inv);
    // (a scalar: with two rows a wavefront it decides over one more per SIMD.  65520 x 1536 into codes 129 -> 125 us)
    if constexpr (T == 64) mean[r].p = __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(mean[r].p)));
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (t + c * T >= n) break;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float x[8];
      unpack8(v[r][c], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) rs[r] = __builtin_fmaf(x[i] - mean[r].p, x[i] - mean[r].p, rs[r]);
    }
  }
  sums(rs, red[1]);
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    rs[r] = row_factor(rs[r] * inv, mean[r].c, a.eps);
    mean[r].c *= -rs[r];                         // (n = (x - p) rs - c rs)
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int e = t + c * T;
    uint4 out[ROWS] = {};
    if (e < n) {
      if constexpr (!EARLY) vectors(c);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        float x[8], u[8];
        unpack8(v[r][c], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(x[i] - mean[r].p, rs[r], mean[r].c);
        if (a.w) {
          unpack8(w[c], u);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= u[i];
        }
        if (a.b) {
          unpack8(b[c], u);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] += u[i];
        }
        if (a.scale.v) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(x[i], sc[c][i], x[i]);
        }
        if (a.shift.v) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] += sh[c][i];
        }
        out[r] = pack8(x);
      }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if constexpr (MX) {
        if (e < mx_steps(a.K) * (MX_STEP / 8) && there(r)) mx_store8(out[r], (int)row(r), e, mx_rows(a.M), a.codes, a.exps);
      } else {
        if (e < n && there(r)) store_to<NT>(share_of(a.y + row(r) * K, e), out[r]);
      }
    }
  }
}

// dx, dres, and each workgroup's shares of the sums over a sample's rows: S0 of dy, S1 of dy o n, S2 of dx o res, each
// [workgroups, K] (all other sums over rows follow from these three: dw = (1 + scale) S1, db = (1 + scale) S0, dscale = w S1 + b S0,
// dshift = S0, dgate = S2).  Workgroup s * chunks + j takes rows j * per .. of sample s.
template <int T, int CH, bool GATE, bool NT>
__global__ void __launch_bounds__(T == 64 ? 256 : T) layer_bwd_kernel(LayerBwdArgs a, int chunks, int per, float* s0, float* s1,
                                                                       float* s2) {
  __shared__ float red[T / 64], red3[3][T / 64];
  __shared__ float4 join[T == 64 ? 6 * CH * 64 : 1];
  constexpr int TEAMS = T == 64 ? 4 : 1;
  // What every row of the sample is multiplied with, (1 + scale) w and the gate, in LDS, each in two halves (no bank twice): in registers
  // it would be 16 a share, and one wavefront per SIMD less.
  // AHEAD: the next row is requested while this one is worked on, where there are registers for it (20000 x 4096 234 -> 219 us; three shares
  // with a gate would have one wavefront per SIMD less: 65520 x 1536 256 -> 267).
  constexpr bool AHEAD = T <= 512 && (CH <= 2 || (CH == 3 && !GATE));
  __shared__ float4 up[2 * T * CH], gates[GATE ? 2 * T * CH : 1];
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = a.K / 8;
  const long long K = a.K;
  const float inv = 1.0f / (float)a.K;
  const int s = blockIdx.x / chunks, j = blockIdx.x - s * chunks;
  const long long first = (long long)s * a.rows + (long long)j * per;
  const long long last = min((long long)a.M, min((long long)(s + 1) * a.rows, first + per));
  for (int e = threadIdx.x; e < n; e += TEAMS * T) {
    float v[8], u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    if (a.scale.v) {
      load8(a.scale.v + s * a.scale.stride + 8 * e, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += u[i];
    }
    if (a.w) {
      unpack8(*(const uint4*)(a.w + 8 * e), u);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= u[i];
    }
    up[e] = float4{v[0], v[1], v[2], v[3]};
    up[T * CH + e] = float4{v[4], v[5], v[6], v[7]};
    if constexpr (GATE) {
      load8(a.gate.v + s * a.gate.stride + 8 * e, v);
      gates[e] = float4{v[0], v[1], v[2], v[3]};
      gates[T * CH + e] = float4{v[4], v[5], v[6], v[7]};
    }
  }
  __syncthreads();
  float a0[CH][8] = {}, a1[CH][8] = {}, a2[GATE ? CH : 1][8] = {};
  struct Row { uint4 g[CH], x[CH], h[CH], r[CH]; };
  auto load = [&](long long m, Row& w) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      w.g[c] = w.x[c] = w.h[c] = w.r[c] = uint4{0u, 0u, 0u, 0u};
      if (t + c * T < n) {
        w.g[c] = load_from<NT, uint4>(share_of(a.dy + m * K, t + c * T));
        w.x[c] = load_from<NT, uint4>(share_of(a.h + m * K, t + c * T));
        if (a.dh) w.h[c] = load_from<NT, uint4>(share_of(a.dh + m * K, t + c * T));
        if (GATE && a.res) w.r[c] = load_from<NT, uint4>(share_of(a.res + m * K, t + c * T));
      }
    }
  };
  auto row = [&](long long m, Row& w, Row& ahead) __attribute__((always_inline)) {
    uint4 (&rg)[CH] = w.g, (&rx)[CH] = w.x, (&rh)[CH] = w.h, (&rr)[CH] = w.r;
    if (AHEAD && m + TEAMS < last) load(m + TEAMS, ahead);
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float x[8];
      unpack8(rx[c], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i];
    }
    const RowMean mean = row_mean(team_sum<T>(sum, red), (float)a.K, inv);
    auto unpack4 = [](uint32_t lo, uint32_t hi, float (&v)[4]) __attribute__((always_inline)) {
      v[0] = bf16_lo(lo); v[1] = bf16_hi(lo); v[2] = bf16_lo(hi); v[3] = bf16_hi(hi);
    };
    auto held = [&](const float4* from, int c, int q, float (&v)[4]) __attribute__((always_inline)) {
      const float4 x = from[q * T * CH + t + c * T];
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    };
    // of half a share: h - p, dy, and g = dy o (1 + scale) o w
    auto half = [&](int c, int q, float (&x)[4], float (&y)[4], float (&g)[4]) __attribute__((always_inline)) {
      float u[4];
      held(up, c, q, u);
      // (formed anew from the packed words each time: kept, they would be 16 registers a share)
      if (q == 0) {
        asm volatile("" : "+v"(rx[c].x), "+v"(rx[c].y), "+v"(rg[c].x), "+v"(rg[c].y));
        unpack4(rx[c].x, rx[c].y, x);
        unpack4(rg[c].x, rg[c].y, y);
      } else {
        asm volatile("" : "+v"(rx[c].z), "+v"(rx[c].w), "+v"(rg[c].z), "+v"(rg[c].w));
        unpack4(rx[c].z, rx[c].w, x);
        unpack4(rg[c].z, rg[c].w, y);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] -= mean.p;
        g[i] = y[i] * u[i];
      }
    };
    float ss = 0.f, sg = 0.f, xg = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (t + c * T >= n) break;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float x[4], y[4], g[4];
        half(c, q, x, y, g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ss = __builtin_fmaf(x[i], x[i], ss);
          sg += g[i];
          xg = __builtin_fmaf(x[i], g[i], xg);
        }
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
    // dx = dh + r (g - mean(g) - n mean(n g)), n = (h - p) r - c r
    const float mg = sg * inv, r = row_factor(ss * inv, mean.c, a.eps), off = -mean.c * r, dot = __builtin_fmaf(-mean.c, mg, xg * inv) * r;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int e = t + c * T;
      if (e >= n) break;
      uint32_t dx[4], dr[4];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float x[4], y[4], g[4], d[4];
        half(c, q, x, y, g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = __builtin_fmaf(x[i], r, off);
          a0[c][4 * q + i] += y[i];
          a1[c][4 * q + i] = __builtin_fmaf(y[i], x[i], a1[c][4 * q + i]);
        }
        unpack4(q ? rh[c].z : rh[c].x, q ? rh[c].w : rh[c].y, d);
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = __builtin_fmaf(__builtin_fmaf(-x[i], dot, g[i] - mg), r, d[i]);
        dx[2 * q] = pack_bf16x2(d[0], d[1]);
        dx[2 * q + 1] = pack_bf16x2(d[2], d[3]);
        if constexpr (GATE) {
          unpack4(q ? rr[c].z : rr[c].x, q ? rr[c].w : rr[c].y, y);
          held(gates, c, q, g);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            a2[c][4 * q + i] = __builtin_fmaf(d[i], y[i], a2[c][4 * q + i]);
            d[i] *= g[i];
          }
          dr[2 * q] = pack_bf16x2(d[0], d[1]);
          dr[2 * q + 1] = pack_bf16x2(d[2], d[3]);
        }
        }
      store_to<NT>(share_of(a.dx + m * K, e), uint4{dx[0], dx[1], dx[2], dx[3]});
      if constexpr (GATE)
        if (a.dres) store_to<NT>(share_of(a.dres + m * K, e), uint4{dr[0], dr[1], dr[2], dr[3]});
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  Row r0, r1;
  long long m = first + (T == 64 ? wave : 0);
  if (AHEAD && m < last) load(m, r0);
  for (; m < last; m += AHEAD ? 2 * TEAMS : TEAMS) {
    if (!AHEAD) load(m, r0);
    row(m, r0, r1);
    if (!AHEAD) continue;
    if (m + TEAMS >= last) break;
    row(m + TEAMS, r1, r0);
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

__device__ __forceinline__ void add4(float4& a, const float4& b) { a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; }
// The gradients that the sums of sample s give in columns x .. x + 3: its vectors' are stored, what it adds to dw and db returned.
__device__ __forceinline__ void layer_grads4(const LayerBwdArgs& a, int s, int x, const float4 (&sum)[3], float4& dw, float4& db) {
  const long long at = (long long)s * a.K + x;
  const float v0[4] = {sum[0].x, sum[0].y, sum[0].z, sum[0].w}, v1[4] = {sum[1].x, sum[1].y, sum[1].z, sum[1].w};
  float up[4] = {1.f, 1.f, 1.f, 1.f}, w[4] = {1.f, 1.f, 1.f, 1.f}, b[4] = {}, ds[4];
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
  for (int i = 0; i < 4; ++i) ds[i] = __builtin_fmaf(w[i], v1[i], b[i] * v0[i]);
  if (a.grads.shift) *(float4*)(a.grads.shift + at) = sum[0];
  if (a.grads.scale) *(float4*)(a.grads.scale + at) = float4{ds[0], ds[1], ds[2], ds[3]};
  if (a.grads.gate) *(float4*)(a.grads.gate + at) = sum[2];
  dw = float4{up[0] * v1[0], up[1] * v1[1], up[2] * v1[2], up[3] * v1[3]};
  db = float4{up[0] * v0[0], up[1] * v0[1], up[2] * v0[2], up[3] * v0[3]};
}

// A sample's sums from its workgroups' shares, in a fixed order, and the gradients they give: workgroup (sample, 64 columns),
// 16 threads of four adjacent columns, 64 along the shares: bound by the latency of a few rounds of loads.  With several samples, what
// each adds to dw and db goes to pw, pb [samples, K], which launch_sum_partials adds up.
constexpr int LSUM_ENTRIES = 64;
__global__ void __launch_bounds__(1024) layer_sums_kernel(LayerBwdArgs a, int chunks, const float* s0, const float* s1,
                                                          const float* s2, float* pw, float* pb) {
  __shared__ float4 red[3][64][16];
  const int blocks = (a.K + LSUM_ENTRIES - 1) / LSUM_ENTRIES, s = blockIdx.x / blocks;
  const int t = threadIdx.x, col = t & 15, row = t >> 4, x = (blockIdx.x - s * blocks) * LSUM_ENTRIES + 4 * col;
  const float* src[3] = {s0, s1, s2};
  float4 v[3] = {};
  if (x < a.K) {
    for (int p = row; p < chunks; p += 128) {
      float4 u[3][2] = {};
      const bool two = p + 64 < chunks;
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        if (!src[k]) continue;
        const float* part = src[k] + ((long long)s * chunks + p) * a.K + x;
        u[k][0] = *(const float4*)part;
        if (two) u[k][1] = *(const float4*)(part + 64ll * a.K);
      }
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        add4(u[k][0], u[k][1]);
        add4(v[k], u[k][0]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) red[k][row][col] = v[k];
  __syncthreads();
  if (row < 48) {                             // kind row / 16: rows r, r + 16, r + 32, r + 48 into row r
    const int k = row >> 4, r = row & 15;
    float4 w = red[k][r][col], y = red[k][r + 32][col];
    add4(w, red[k][r + 16][col]);
    add4(y, red[k][r + 48][col]);
    add4(w, y);
    red[k][r][col] = w;
  }
  __syncthreads();
  if (row < 12) {
    const int k = row >> 2, r = row & 3;
    float4 w = red[k][r][col], y = red[k][r + 8][col];
    add4(w, red[k][r + 4][col]);
    add4(y, red[k][r + 12][col]);
    add4(w, y);
    red[k][r][col] = w;
  }
  __syncthreads();
  if (t >= 16 || x >= a.K) return;
  float4 sum[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    sum[k] = red[k][0][t];
    float4 y = red[k][2][t];
    add4(sum[k], red[k][1][t]);
    add4(y, red[k][3][t]);
    add4(sum[k], y);
  }
  float4 dw, db;
  layer_grads4(a, s, x, sum, dw, db);
  const long long at = (long long)s * a.K + x;
  if (pw) *(float4*)(pw + at) = dw;
  if (pb) *(float4*)(pb + at) = db;
}

// The same where a sample has few shares (many samples, down to a modulation of each row): four columns a thread, every `parts`-th
// sample, whose additions to dw and db it adds up on the way (pw, pb [parts, K]).
constexpr int LSUM_COLUMNS = 1024;
__global__ void __launch_bounds__(256) layer_samples_kernel(LayerBwdArgs a, int samples, int chunks, int parts, const float* s0,
                                                            const float* s1, const float* s2, float* pw, float* pb) {
  const int blocks = (a.K + LSUM_COLUMNS - 1) / LSUM_COLUMNS, part = blockIdx.x / blocks;
  const int x = (blockIdx.x - part * blocks) * LSUM_COLUMNS + 4 * threadIdx.x;
  if (x >= a.K) return;
  const float* src[3] = {s0, s1, s2};
  float4 dw{}, db{};
  for (int s = part; s < samples; s += parts) {
    float4 sum[3] = {}, w, b;
    for (int p = 0; p < chunks; ++p)
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (src[k]) add4(sum[k], *(const float4*)(src[k] + ((long long)s * chunks + p) * a.K + x));
    layer_grads4(a, s, x, sum, w, b);
    add4(dw, w);
    add4(db, b);
  }
  const long long at = (long long)part * a.K + x;
  if (pw) *(float4*)(pw + at) = dw;
  if (pb) *(float4*)(pb + at) = db;
}

// ---------------------------------------------------------------------------
// The team and the shares of a thread for n shares of eight features: F(T, CH).  Forward a wavefront per row up to K = 2048 (nothing
// is exchanged), above that workgroups of two shares a thread, whose size follows the width so that few threads idle (20000 x 8960 277 -> 257 us
// against 1024 threads from K = 8200 on, into codes 261 -> 230).  Backward the sums cost 8 to 24 registers a share: without a gate three shares
// of 768 threads at most, with one four of 512 (20000 x 13824 838 -> 659 us, without a gate 474 -> 456, against 1024 threads of two).
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
    else if (n_ <= 1280) F(640, 2);       \
    else if (n_ <= 1536) F(768, 2);       \
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
    else if (gate) F(512, 4);             \
    else F(768, 3);                       \
  } while (0)

// `tensors` of these that do not fit the memory-side cache (256 MiB) together are read and written past it.
static bool streams(int M, int K, int tensors) { return (long long)M * K * 2 * tensors > (256ll << 20); }

void launch_layer_fwd(const LayerArgs& a, hipStream_t stream) {
  const bool nt = streams(a.M, a.K, a.res ? 4 : 2);
  const int rows = min(a.rows, a.M);
  // Two rows at a time share the vectors (75600 x 5120 601 -> 541 us, 20000 x 8192 256 -> 232, 20000 x 13824 414 -> 404), where there are so many
  // that the chip is full all the same (1000 x 5120 11.5 / 12.2, 1000 x 1536 6.6 / 7.8); a wavefront's rows only on their way into codes, two of
  // which are a line (65520 x 1536 -> 8960 612 -> 598; 65520 x 1536 by itself 141 / 143), and millions of any rows (2500000 x 520 1073 -> 1048,
  // 2500000 x 5120 8810 -> 8660).
  const bool two = rows > 1 && a.M >= 4096 && (a.codes || (a.K > 2048 && (a.gate.v || a.scale.v || a.shift.v)) || a.M > (1 << 21));
  const int per_sample = two ? (rows + 1) / 2 : rows, whole = a.M / rows, left = a.M - whole * rows;
  const int groups = whole * per_sample + (two ? (left + 1) / 2 : left);
  // A row of a grid has fewer than 2^32 threads: 2^22 teams of 1024 take two.
  auto grid = [&](int T) {
    const unsigned n = (unsigned)(T == 64 ? (groups + 3) / 4 : groups);
    return (unsigned long long)n * T >> 32 ? dim3((n + 1) / 2, 2) : dim3(n);
  };
#define LAYER_FWD_(T, CH, ROWS, MX, NT) \
  layer_fwd_kernel<T, CH, ROWS, MX, NT><<<grid(T), T == 64 ? 256 : T, 0, stream>>>(a, groups, per_sample)
#define LAYER_FWD(T, CH)                                                                                       \
  do {                                                                                                         \
    if (a.codes) {                                                                                             \
      if (two) { if (nt) LAYER_FWD_(T, CH, 2, true, true); else LAYER_FWD_(T, CH, 2, true, false); }           \
      else { if (nt) LAYER_FWD_(T, CH, 1, true, true); else LAYER_FWD_(T, CH, 1, true, false); }               \
    } else {                                                                                                   \
      if (two) { if (nt) LAYER_FWD_(T, CH, 2, false, true); else LAYER_FWD_(T, CH, 2, false, false); }         \
      else { if (nt) LAYER_FWD_(T, CH, 1, false, true); else LAYER_FWD_(T, CH, 1, false, false); }             \
    }                                                                                                          \
  } while (0)
  LAYER_TEAMS(a.codes ? mx_steps(a.K) * (MX_STEP / 8) : a.K / 8, LAYER_FWD);   // (codes: those behind the last feature too)
#undef LAYER_FWD
#undef LAYER_FWD_
}

// How a sample's rows are dealt: at least eight to a workgroup (to a team), but enough workgroups to fill the chip; more of them would only
// leave more shares.  In us with at most 256 / 512 / 1024 workgroups (at least half of that): 1000 x 5120 33.1 / 29.8 / 31.4, 8192 x 5120
// 125 / 116 / 128, 20000 x 5120 271 / 257 / 269, 65520 x 1536 253 / 256 / 250; with 128 / 256 / 512: 2048 x 13824 116 / 96 / 96, 8192 x 13824 395 / 288 /
// 299.
// many: so many samples of so few shares that layer_samples_kernel adds them up (whole backward pass in us, else / so: 300 x 5120 in 100
// samples 57 / 26, 1000 x 1536 in 500 74 / 27, 8000 x 5120 in 64 135 / 121; 8 x 5120, one sample, 10.6 / 15.4); parts: of dw and db, before the
// last step adds them up.
struct LayerDeal { int samples, chunks, per, parts; bool many; };
static LayerDeal layer_deal(int M, int K, int rows) {
  rows = min(rows, M);
  const int samples = (M + rows - 1) / rows, teams = K <= 2048 ? 4 : 1, most = K <= 8192 ? 512 : 256;
  const int all = (rows + teams - 1) / teams;                              // chunks of one row per team
  const int want = max(1, (min(most, max(most / 2, M / (8 * teams))) + samples - 1) / samples);
  const int per = teams * ((all + min(all, want) - 1) / min(all, want));
  const int chunks = (rows + per - 1) / per;
  const bool many = chunks == 1 || (chunks <= 8 && samples >= 32);
  return {samples, chunks, per, many ? min(samples, 2048 / ((K + LSUM_COLUMNS - 1) / LSUM_COLUMNS)) : samples, many};
}
// three sums per workgroup, and the parts of dw and db
size_t layer_bwd_bytes(int M, int K, int rows) {
  const LayerDeal d = layer_deal(M, K, rows);
  return 3 * align256((size_t)d.samples * d.chunks * K * 4) + (d.parts > 1 ? 2 * align256((size_t)d.parts * K * 4) : 0);
}

void launch_layer_bwd(const LayerBwdArgs& a, hipStream_t stream) {
  const LayerDeal d = layer_deal(a.M, a.K, a.rows);
  const norm_layer_grads& g = a.grads;
  const size_t one = align256((size_t)d.samples * d.chunks * a.K * 4), part = align256((size_t)d.parts * a.K * 4);
  unsigned char* ws = (unsigned char*)a.ws;
  const bool sums = g.w || g.b || g.scale || g.shift;
  float *s0 = sums ? (float*)ws : nullptr, *s1 = sums ? (float*)(ws + one) : nullptr, *s2 = g.gate ? (float*)(ws + 2 * one) : nullptr;
  const unsigned grid = (unsigned)d.samples * d.chunks;
  const bool gate = a.gate.v != nullptr, nt = streams(a.M, a.K, 3 + (a.dh != nullptr) + 2 * gate);
#define LAYER_BWD_(T, CH, GATE)                                                                                              \
  do {                                                                                                                       \
    constexpr int threads = T == 64 ? 256 : T;                                                                               \
    if (nt) layer_bwd_kernel<T, CH, GATE, true><<<grid, threads, 0, stream>>>(a, d.chunks, d.per, s0, s1, s2);               \
    else layer_bwd_kernel<T, CH, GATE, false><<<grid, threads, 0, stream>>>(a, d.chunks, d.per, s0, s1, s2);                 \
  } while (0)
#define LAYER_BWD(T, CH)                                                                                                     \
  do {   /* (the widest rows have teams of their own with a gate and without) */                                             \
    if constexpr (T == 512 && CH == 4) LAYER_BWD_(T, CH, true);                                                              \
    else if constexpr (T == 768) LAYER_BWD_(T, CH, false);                                                                   \
    else if (gate) LAYER_BWD_(T, CH, true);                                                                                  \
    else LAYER_BWD_(T, CH, false);                                                                                           \
  } while (0)
  LAYER_BWD_TEAMS(a.K / 8, LAYER_BWD);
#undef LAYER_BWD
#undef LAYER_BWD_
  if (!sums && !g.gate) return;
  float *pw = g.w, *pb = g.b;
  if (d.parts > 1) {
    pw = g.w ? (float*)(ws + 3 * one) : nullptr;
    pb = g.b ? (float*)(ws + 3 * one + part) : nullptr;
  }
  if (d.many)
    layer_samples_kernel<<<(unsigned)d.parts * ((a.K + LSUM_COLUMNS - 1) / LSUM_COLUMNS), 256, 0, stream>>>(a, d.samples, d.chunks, d.parts, s0, s1, s2, pw, pb);
  else
    layer_sums_kernel<<<(unsigned)d.samples * ((a.K + LSUM_ENTRIES - 1) / LSUM_ENTRIES), 1024, 0, stream>>>(a, d.chunks, s0, s1, s2, pw, pb);
  if (d.parts > 1 && (g.w || g.b)) {
    PartialSums p{};
    p.part[0] = pw; p.dw[0] = g.w; p.width[0] = a.K;
    p.part[1] = pb; p.dw[1] = g.b; p.width[1] = a.K;
    p.n_part = d.parts;
    launch_sum_partials(p, stream);
  }
}

}  // namespace sla
