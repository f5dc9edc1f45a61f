// Rotary positions over several axes with the root-mean-square norm of queries and keys (include/rope.h), forward and
// backward.
//
//   rope_fwd_kernel       a team of threads per token: reads the token's q and k once, norms, turns, writes once.
//   rope_bwd_kernel       the same for the gradients; teams walk over the tokens and keep their share of the weight's gradient
//                         in registers.
//   sum_partials_kernel   joins those shares in a fixed order.
//
// Bound by HBM: 2 bytes per element and tensor read or written.  75600 tokens of 40 heads, q and k, normed over the token: forward 519
// us token-major (6.0 TB/s), 630 head-major (256 bytes at a time to 80 places); backward 956 (4.9).  32760 of 12: 67 and 121.  A thread holds 8 channels, four whole pairs, of head
// e / 16 for e = its number + T c; a head is 16 lanes, so a head's sums stay in a row of lanes.  The 64 angles of a token
// are one per lane of a wavefront: each lane forms one sine and cosine, and the lanes fetch the four pairs they turn from LDS.
#include "rows.h"

namespace sla {

// cos and sin of a full turn's fraction t / 2^64.  The nearest multiple of a quarter is taken off in integers; what is left,
// at most an eighth of a turn, goes through the Taylor polynomials (next terms: x^11 / 11! = 1.8e-9, x^12 / 12! = 1.2e-10 of
// x = pi / 4: below half a step of fp32).
__device__ __forceinline__ float2 cos_sin(uint64_t t) {
  const uint32_t a = (uint32_t)((t + 0x80000000ull) >> 32);
  const uint32_t quarter = (a + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(a - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi 2^-32
  const float x2 = x * x;
  float s = __builtin_fmaf(x2, 2.7557319e-6f, -1.9841270e-4f);
  s = __builtin_fmaf(x2, s, 8.3333333e-3f);
  s = __builtin_fmaf(x2, s, -1.6666667e-1f);
  s = __builtin_fmaf(x * x2, s, x);
  float c = __builtin_fmaf(x2, -2.7557319e-7f, 2.4801587e-5f);
  c = __builtin_fmaf(x2, c, -1.3888889e-3f);
  c = __builtin_fmaf(x2, c, 4.1666667e-2f);
  c = __builtin_fmaf(x2, c, -0.5f);
  c = __builtin_fmaf(x2, c, 1.0f);
  const float cs = (quarter & 1) ? s : c, sn = (quarter & 1) ? c : s;
  return float2{((quarter + 1) & 2) ? -cs : cs, (quarter & 2) ? -sn : sn};
}

// A token's angles to a wavefront's 64 entries of LDS, then the four of this lane's pairs (4 part .. 4 part + 3).
__device__ __forceinline__ void token_angles(const RopeArgs& a, int b, int n, float2* mine, int lane, float2 (&cs)[4]) {
  const int32_t p = a.pos[b * a.pos_batch + 3ll * n + a.plan.axis[lane]];
  __builtin_amdgcn_wave_barrier();      // (a wavefront's LDS operations execute in order: only the compiler has to keep it)
  mine[lane] = cos_sin((uint64_t)(int64_t)p * a.plan.turns[lane]);
  __builtin_amdgcn_wave_barrier();
  const int part = lane & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i) cs[i] = mine[4 * part + i];
}

// Four pairs of a head: the words of part `part` of its 256 bytes, and their numbers lo[i], hi[i].
template <bool HALVES, bool NT>
__device__ __forceinline__ uint4 load_pairs(const bf16_t* head, int part) {
  if constexpr (!HALVES) return load_from<NT, uint4>(head + 8 * part);
  const uint2 lo = load_from<NT, uint2>(head + 4 * part), hi = load_from<NT, uint2>(head + D / 2 + 4 * part);
  return uint4{lo.x, lo.y, hi.x, hi.y};
}
template <bool HALVES, bool NT>
__device__ __forceinline__ void store_pairs(bf16_t* head, int part, const uint4& v) {
  if constexpr (!HALVES) {
    store_to<NT>(head + 8 * part, v);
  } else {
    store_to<NT>(head + 4 * part, uint2{v.x, v.y});
    store_to<NT>(head + D / 2 + 4 * part, uint2{v.z, v.w});
  }
}
template <bool HALVES>
__device__ __forceinline__ void unpack_pairs(const uint4& v, float (&lo)[4], float (&hi)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (!HALVES) {
      lo[i] = bf16_lo(w[i]);
      hi[i] = bf16_hi(w[i]);
    } else {
      lo[i] = (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
      hi[i] = (i & 1) ? bf16_hi(w[2 + (i >> 1)]) : bf16_lo(w[2 + (i >> 1)]);
    }
  }
}
template <bool HALVES>
__device__ __forceinline__ uint4 pack_pairs(const float (&lo)[4], const float (&hi)[4]) {
  if constexpr (!HALVES)
    return uint4{pack_bf16x2(lo[0], hi[0]), pack_bf16x2(lo[1], hi[1]), pack_bf16x2(lo[2], hi[2]), pack_bf16x2(lo[3], hi[3])};
  return uint4{pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
}
// A norm's weights for head `head`: ones without.
template <int NORM, bool HALVES>
__device__ __forceinline__ void weight_pairs(const bf16_t* w, int head, int part, float (&lo)[4], float (&hi)[4]) {
  if (w) {
    unpack_pairs<HALVES>(load_pairs<HALVES, false>(w + (NORM == 2 ? head * D : 0), part), lo, hi);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) lo[i] = hi[i] = 1.0f;
  }
}
__device__ __forceinline__ float pair_dot(const float (&al)[4], const float (&ah)[4], const float (&bl)[4], const float (&bh)[4]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) s = __builtin_fmaf(al[i], bl[i], __builtin_fmaf(ah[i], bh[i], s));
  return s;
}

// NORM: rope_norm.  T: threads of a team (64: up to 16 heads, 256: up to 64); CH: a thread's shares of a token.
template <int T, int CH, int NORM, bool HALVES, bool NT>
__global__ void __launch_bounds__(256) rope_fwd_kernel(RopeArgs a) {
  __shared__ float2 angles[4][64];
  __shared__ float red[2][4];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, part = lane & 15, e0 = (T == 64 ? lane : t) >> 4;
  const int tok = T == 64 ? 4 * blockIdx.x + w : blockIdx.x;                 // (below 2^24)
  if (T == 64 && tok >= a.B * a.N) return;
  const int b = tok / a.N, n = tok - b * a.N;
  uint4 raw[2][CH];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const RopeTensor& x = a.t[i];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int head = e0 + c * (T / 16);
      raw[i][c] = uint4{0u, 0u, 0u, 0u};
      if (head < x.H) raw[i][c] = load_pairs<HALVES, NT>(x.x + b * x.lx.sb + head * x.lx.sh + n * x.lx.sn, part);
    }
  }
  float2 cs[4];
  token_angles(a, b, n, angles[w], lane, cs);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const RopeTensor& x = a.t[i];
    if (x.H == 0) break;
    float r = 1.0f;
    if constexpr (NORM == 2) {
      float ss = 0.f;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        float lo[4], hi[4];
        unpack_pairs<HALVES>(raw[i][c], lo, hi);
        ss += pair_dot(lo, hi, lo, hi);
      }
      r = __builtin_amdgcn_rsqf(team_sum<T>(ss, red[i]) / (float)(x.H * D) + a.eps);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int head = e0 + c * (T / 16);
      float lo[4], hi[4];
      unpack_pairs<HALVES>(raw[i][c], lo, hi);
      if constexpr (NORM == 1) r = __builtin_amdgcn_rsqf(row_sum(pair_dot(lo, hi, lo, hi)) * (1.0f / D) + a.eps);
      if (head >= x.H) break;
      if constexpr (NORM != 0) {
        float wl[4], wh[4];
        weight_pairs<NORM, HALVES>(x.w, head, part, wl, wh);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          lo[j] = lo[j] * r * wl[j];
          hi[j] = hi[j] * r * wh[j];
        }
      }
      float yl[4], yh[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        yl[j] = __builtin_fmaf(lo[j], cs[j].x, -hi[j] * cs[j].y);
        yh[j] = __builtin_fmaf(lo[j], cs[j].y, hi[j] * cs[j].x);
      }
      store_pairs<HALVES, NT>(x.y + b * x.ly.sb + head * x.ly.sh + n * x.ly.sn, part, pack_pairs<HALVES>(yl, yh));
    }
  }
}

// Gradients, blockIdx.y: q or k.  Each team takes every (teams)-th token.
template <int T, int CH, int NORM, bool HALVES, bool NT>
__global__ void __launch_bounds__(256) rope_bwd_kernel(RopeArgs a) {
  __shared__ float2 angles[4][64];
  __shared__ float red[2][4];
  constexpr int ACC = NORM == 0 ? 1 : NORM == 1 ? 1 : CH;    // shares of the weight's gradient (a head's weight: one for all)
  __shared__ float4 join[NORM == 0 ? 1 : ACC * 2 * 64];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, part = lane & 15, e0 = (T == 64 ? lane : t) >> 4;
  const RopeTensor& x = a.t[blockIdx.y];
  const int tokens = a.B * a.N;                // (below 2^24)
  const float inv = NORM == 2 ? 1.0f / (float)(x.H * D) : 1.0f / D;
  float dwl[ACC][4] = {}, dwh[ACC][4] = {};
  int turn = 0;
  for (int tok = T == 64 ? 4 * blockIdx.x + w : blockIdx.x; tok < tokens; tok += gridDim.x * (256 / T), turn ^= 1) {
    const int b = tok / a.N, n = tok - b * a.N;
    uint4 rg[CH], rx[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int head = e0 + c * (T / 16);
      rg[c] = rx[c] = uint4{0u, 0u, 0u, 0u};
      if (head < x.H) {
        rg[c] = load_pairs<HALVES, NT>(x.dy + b * x.ldy.sb + head * x.ldy.sh + n * x.ldy.sn, part);
        if constexpr (NORM != 0) rx[c] = load_pairs<HALVES, NT>(x.x + b * x.lx.sb + head * x.lx.sh + n * x.lx.sn, part);
      }
    }
    float2 cs[4];
    token_angles(a, b, n, angles[w], lane, cs);
    // the output's gradient turned back
    auto back = [&](int c, float (&gl)[4], float (&gh)[4]) __attribute__((always_inline)) {
      float yl[4], yh[4];
      unpack_pairs<HALVES>(rg[c], yl, yh);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        gl[j] = __builtin_fmaf(yl[j], cs[j].x, yh[j] * cs[j].y);
        gh[j] = __builtin_fmaf(yh[j], cs[j].x, -yl[j] * cs[j].y);
      }
    };
    auto put = [&](int head, const float (&gl)[4], const float (&gh)[4]) __attribute__((always_inline)) {
      store_pairs<HALVES, NT>(x.y + b * x.ly.sb + head * x.ly.sh + n * x.ly.sn, part, pack_pairs<HALVES>(gl, gh));
    };
    float r = 1.0f, dot = 0.f;
    if constexpr (NORM == 2) {
      float ss = 0.f, xg = 0.f;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int head = min(e0 + c * (T / 16), x.H - 1);    // (beyond: x and g are zero)
        float xl[4], xh[4], gl[4], gh[4], wl[4], wh[4];
        unpack_pairs<HALVES>(rx[c], xl, xh);
        back(c, gl, gh);
        weight_pairs<NORM, HALVES>(x.w, head, part, wl, wh);
        ss += pair_dot(xl, xh, xl, xh);
#pragma unroll
        for (int j = 0; j < 4; ++j) xg = __builtin_fmaf(xl[j] * wl[j], gl[j], __builtin_fmaf(xh[j] * wh[j], gh[j], xg));
      }
      if constexpr (T == 64) {
        ss = team_sum<T>(ss, red[0]);
        xg = team_sum<T>(xg, red[1]);
      } else {                                               // (both sums behind one barrier)
        __shared__ float red2[2][2][4];
        ss = rows_sum(row_sum(ss));
        xg = rows_sum(row_sum(xg));
        if (lane == 0) { red2[turn][0][w] = ss; red2[turn][1][w] = xg; }
        __syncthreads();
        ss = red2[turn][0][0] + red2[turn][0][1] + red2[turn][0][2] + red2[turn][0][3];
        xg = red2[turn][1][0] + red2[turn][1][1] + red2[turn][1][2] + red2[turn][1][3];
      }
      r = __builtin_amdgcn_rsqf(ss * inv + a.eps);
      dot = xg * inv * r * r;            // (dx = r (w g - x r^2 mean(x w g)): r^3 need not be a number of fp32)
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int head = e0 + c * (T / 16);
      float gl[4], gh[4];
      back(c, gl, gh);
      if constexpr (NORM != 0) {
        float xl[4], xh[4], wl[4], wh[4];
        unpack_pairs<HALVES>(rx[c], xl, xh);
        weight_pairs<NORM, HALVES>(x.w, min(head, x.H - 1), part, wl, wh);
        if constexpr (NORM == 1) {
          float xg = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) xg = __builtin_fmaf(xl[j] * wl[j], gl[j], __builtin_fmaf(xh[j] * wh[j], gh[j], xg));
          r = __builtin_amdgcn_rsqf(row_sum(pair_dot(xl, xh, xl, xh)) * inv + a.eps);
          dot = row_sum(xg) * inv * r * r;
        }
        const int u = NORM == 1 ? 0 : c;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          dwl[u][j] = __builtin_fmaf(gl[j] * xl[j], r, dwl[u][j]);
          dwh[u][j] = __builtin_fmaf(gh[j] * xh[j], r, dwh[u][j]);
          gl[j] = __builtin_fmaf(-xl[j], dot, gl[j] * wl[j]) * r;
          gh[j] = __builtin_fmaf(-xh[j], dot, gh[j] * wh[j]) * r;
        }
      }
      if (head < x.H) put(head, gl, gh);
    }
  }
  if constexpr (NORM != 0) {
    if (!x.part) return;
    // channels of lo[j], hi[j]: 2 (4 part + j), + 1, or 4 part + j and 64 on
    auto store = [&](float* head, const float (&l)[4], const float (&h)[4]) __attribute__((always_inline)) {
      if constexpr (HALVES) {
        *(float4*)(head + 4 * part) = float4{l[0], l[1], l[2], l[3]};
        *(float4*)(head + D / 2 + 4 * part) = float4{h[0], h[1], h[2], h[3]};
      } else {
        *(float4*)(head + 8 * part) = float4{l[0], h[0], l[1], h[1]};
        *(float4*)(head + 8 * part + 4) = float4{l[2], h[2], l[3], h[3]};
      }
    };
    if constexpr (NORM == 1) {
      // one head's weight: over the heads that share a lane row (rows of a wavefront), then over the wavefronts
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        dwl[0][j] = rows_sum(dwl[0][j]);
        dwh[0][j] = rows_sum(dwh[0][j]);
      }
    }
    if constexpr (T == 64 || NORM == 1) {                    // four wavefronts hold shares of the same channels
      for (int k = 0; k < 4; ++k) {
        if (w == k) {
#pragma unroll
          for (int u = 0; u < ACC; ++u) {
            float4 l{dwl[u][0], dwl[u][1], dwl[u][2], dwl[u][3]}, h{dwh[u][0], dwh[u][1], dwh[u][2], dwh[u][3]};
            if (k > 0) {
              const float4 pl = join[(2 * u) * 64 + lane], ph = join[(2 * u + 1) * 64 + lane];
              l.x += pl.x; l.y += pl.y; l.z += pl.z; l.w += pl.w;
              h.x += ph.x; h.y += ph.y; h.z += ph.z; h.w += ph.w;
            }
            join[(2 * u) * 64 + lane] = l;
            join[(2 * u + 1) * 64 + lane] = h;
          }
        }
        __syncthreads();
      }
      if (w == 0) {
#pragma unroll
        for (int u = 0; u < ACC; ++u) {
          const float4 l = join[(2 * u) * 64 + lane], h = join[(2 * u + 1) * 64 + lane];
          const float sl[4] = {l.x, l.y, l.z, l.w}, sh[4] = {h.x, h.y, h.z, h.w};
          const int head = NORM == 1 ? 0 : e0 + u * (T / 16);
          if (NORM == 1 ? lane < 16 : head < x.H)
            store(x.part + (long long)blockIdx.x * (NORM == 1 ? D : x.H * D) + (NORM == 1 ? 0 : head * D), sl, sh);
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < ACC; ++u) {
        const int head = e0 + u * (T / 16);
        if (head < x.H) store(x.part + (long long)blockIdx.x * (x.H * D) + head * D, dwl[u], dwh[u]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
constexpr int SUM_ENTRIES = 64;   // columns of a workgroup: 16 threads of four, 16 threads along the partials
__global__ void __launch_bounds__(256) sum_partials_kernel(PartialSums s) {
  __shared__ float4 red[16][16];
  const float* part = s.part[blockIdx.y];
  const int width = s.width[blockIdx.y], t = threadIdx.x, col = t & 15, row = t >> 4;
  const int x = blockIdx.x * SUM_ENTRIES + 4 * col;
  if (!part) return;
  auto add = [](float4& a, const float4& b) __attribute__((always_inline)) { a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; };
  float4 v[4] = {};
  if (x < width) {
    int p = row;
    for (; p + 48 < s.n_part; p += 64)
#pragma unroll
      for (int u = 0; u < 4; ++u) add(v[u], *(const float4*)(part + (long long)(p + 16 * u) * width + x));
    for (; p < s.n_part; p += 16) add(v[0], *(const float4*)(part + (long long)p * width + x));
  }
  add(v[0], v[1]);
  add(v[2], v[3]);
  add(v[0], v[2]);
  red[row][col] = v[0];
  __syncthreads();
  if (t < 16 && x < width) {
    float4 r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = red[i][t];
#pragma unroll
    for (int step = 1; step < 16; step *= 2)
#pragma unroll
      for (int i = 0; i < 16; i += 2 * step) add(r[i], r[i + step]);
    float* to = s.dw[blockIdx.y] + x;      // (a caller's tensor may start at any element)
    to[0] = r[0].x; to[1] = r[0].y; to[2] = r[0].z; to[3] = r[0].w;
  }
}
void launch_sum_partials(const PartialSums& s, hipStream_t stream) {
  const int width = max(s.part[0] ? s.width[0] : 0, s.part[1] ? s.width[1] : 0);
  if (width == 0) return;
  sum_partials_kernel<<<dim3((unsigned)((width + SUM_ENTRIES - 1) / SUM_ENTRIES), 2), 256, 0, stream>>>(s);
}

// ---------------------------------------------------------------------------
// The call's tensors do not fit the memory-side cache: they are read and written past it (75600 x 40 heads, token-major, forward
// 568 -> 516 us without a norm, 543 -> 536 with one over the token; 32760 x 12 78 -> 66); where they fit, that costs (4096 x 24 heads,
// the norm over the token 20 -> 23 us).
static bool streams(const RopeArgs& a, bool bwd) {
  const long long elems = (long long)a.B * a.N * (a.t[0].H + a.t[1].H) * D;
  return elems * 2 * (bwd && a.t[0].x ? 3 : 2) > (256ll << 20);
}
template <int T, int CH, int NORM, bool HALVES, bool NT>
static void launch_rope(const RopeArgs& a, bool bwd, hipStream_t stream) {
  const long long tokens = (long long)a.B * a.N;
  if (bwd) {
    // (without a weight to sum up for there is nothing to walk for: 75600 x 40 heads 643 us with 512 workgroups, 617 with 2048)
    const int heads = max(a.t[0].H, a.t[1].H), groups = NORM == 0 ? (int)min((tokens * T + 255) / 256, 1ll << 16) : rope_bwd_workgroups(tokens, heads);
    rope_bwd_kernel<T, CH, NORM, HALVES, NT><<<dim3((unsigned)groups, a.t[1].H ? 2 : 1), 256, 0, stream>>>(a);
  } else {
    rope_fwd_kernel<T, CH, NORM, HALVES, NT><<<(unsigned)(T == 64 ? (tokens + 3) / 4 : tokens), 256, 0, stream>>>(a);
  }
}
template <int T, int CH, int NORM>
static void launch_rope(const RopeArgs& a, bool bwd, bool halves, hipStream_t stream) {
  const bool nt = streams(a, bwd);
  if (halves && nt) launch_rope<T, CH, NORM, true, true>(a, bwd, stream);
  else if (halves) launch_rope<T, CH, NORM, true, false>(a, bwd, stream);
  else if (nt) launch_rope<T, CH, NORM, false, true>(a, bwd, stream);
  else launch_rope<T, CH, NORM, false, false>(a, bwd, stream);
}
template <int T, int CH>
static void launch_rope(const RopeArgs& a, bool bwd, int norm, bool halves, hipStream_t stream) {
  if (norm == 0) launch_rope<T, CH, 0>(a, bwd, halves, stream);
  else if (norm == 1) launch_rope<T, CH, 1>(a, bwd, halves, stream);
  else launch_rope<T, CH, 2>(a, bwd, halves, stream);
}
static void launch_rope(const RopeArgs& a, bool bwd, int norm, bool halves, hipStream_t stream) {
  // Up to 16 heads a wavefront takes a token by itself (at most four shares of 16 bytes per lane); more heads take a workgroup.  The
  // shares are counted in steps of four and of sixteen heads: one count for up to 16 (four) and one beyond (four) cost the gradient
  // registers that hold nothing (norm over the token, us: 32760 tokens of 4 heads 44 -> 91, of 8 84 -> 138, of 12 121 -> 160, of 24 269 ->
  // 482, 75600 of 40 910 -> 1228), the forward direction a little (2 heads 19.5 -> 23.9, 24 heads 137 -> 146), and no norm nothing.
  const int heads = max(a.t[0].H, a.t[1].H);
  if (heads <= 4) launch_rope<64, 1>(a, bwd, norm, halves, stream);
  else if (heads <= 8) launch_rope<64, 2>(a, bwd, norm, halves, stream);
  else if (heads <= 12) launch_rope<64, 3>(a, bwd, norm, halves, stream);
  else if (heads <= 16) launch_rope<64, 4>(a, bwd, norm, halves, stream);
  else if (heads <= 32) launch_rope<256, 2>(a, bwd, norm, halves, stream);
  else if (heads <= 48) launch_rope<256, 3>(a, bwd, norm, halves, stream);
  else launch_rope<256, 4>(a, bwd, norm, halves, stream);
}

// Two to a compute unit and tensor: what it holds (8192 tokens of 24 heads, in us: 128 workgroups 145, 256 90, 512 78; 75600 of 40 heads
// 512 962, 1024 957, 32760 of 12 121 and 125).  The next token's rows requested ahead cost more in wavefronts than they hid
// (75600 of 40 heads 1067 us).
int rope_bwd_workgroups(long long tokens, int heads) {
  const long long all = heads <= 16 ? (tokens + 3) / 4 : tokens;
  return (int)min(all, 512ll);
}
void launch_rope_fwd(const RopeArgs& a, int norm, bool halves, hipStream_t stream) { launch_rope(a, false, norm, halves, stream); }
void launch_rope_bwd(const RopeArgs& a, int norm, bool halves, hipStream_t stream) {
  launch_rope(a, true, norm, halves, stream);
  PartialSums s{};
  s.n_part = rope_bwd_workgroups((long long)a.B * a.N, max(a.t[0].H, a.t[1].H));
  for (int i = 0; i < 2; ++i) {
    s.part[i] = a.t[i].H ? a.t[i].part : nullptr;
    s.dw[i] = a.t[i].dw;
    s.width[i] = norm == 1 ? D : a.t[i].H * D;
  }
  launch_sum_partials(s, stream);
}

}  // namespace sla
