// Attention to a sequence of another length (include/xattn.h), forward and backward.
//
//   xattn_fwd_kernel     per 32 to 128 query rows, over the keys: one pass with a running maximum and sum.
//   xattn_join_kernel    joins the pieces of a walk that was split: weights 2^(m - max m), one division.
//   xattn_dq_kernel      per 32 to 128 query rows, over the keys: delta = dout . out, dQ += dS K; leaves delta for the next one.
//   xattn_dkv_kernel     per 32 to 128 keys, over the query rows of every head that shares them: dV += P^T dO, dK += dS^T Q.
//   xattn_sum_kernel     adds up the pieces of split walks of the two.
//
// All products are formed transposed where that saves a shuffle: a wavefront owns 32 rows, one per lane pair, so a row's
// statistics stay inside the pair, and an accumulator tile converted to bf16 is the B operand of the next product (its
// contraction index = the accumulator's rows).  Tiles of 32 rows are copied to LDS one step ahead (tiles.h).
//
// A key head's query rows are those of all heads that share it, head after head, so that its keys are read once for all of
// them.  Where the rows do not fill the chip (few tokens against a long memory) the walk is split and joined through the
// workspace.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "tiles.h"
#include "xattn.h"

namespace sla {

constexpr int XATTN_PIECES = 1024;             // most pieces of a walk

// Consecutive workgroups go to the eight XCDs in turn: each XCD gets a contiguous eighth of every sample's units, so that the
// workgroups on it at a time work on neighbouring ones (the same slice's keys), and samples of different lengths leave no
// XCD idle (an eighth of all the units: prompts of 512 and 128 states, 12 heads x 32760 queries 226 us, half the XCDs done early;
// so 181; the samples in turn, unit by unit, 165 -> 198 with the present kernel).  Samples of few units, which do not divide by eight, are taken together.  False: no unit.
// (All counts are below 2^31: divisions of 32 bits.)
__host__ __device__ inline unsigned xattn_part(unsigned per_sample, unsigned B) { return per_sample >= 64 ? per_sample : per_sample * B; }
__device__ __forceinline__ bool xattn_unit(unsigned per_sample, unsigned B, unsigned& unit) {
  const unsigned part = xattn_part(per_sample, B), per = (part + 7) >> 3, slot = blockIdx.x >> 3, which = slot / per;
  const unsigned in_part = (blockIdx.x & 7) * per + (slot - which * per);
  unit = which * part + in_part;
  return in_part < part && unit < per_sample * B;
}
// Numbers of workgroups that have a unit, and some that have none.
__host__ __device__ inline unsigned xattn_numbers(unsigned per_sample, unsigned B) {
  const unsigned part = xattn_part(per_sample, B);
  return 8 * ((part + 7) / 8) * (per_sample * B / part);
}

// TileCopy for rows that are 16-byte aligned whatever the strides are.
template <int WAVES>
struct AlignedCopy : TileCopy<WAVES> {
  template <bool ZEROS = false>
  __device__ __forceinline__ void tile(int row0, int N, unsigned lds_tile) const {
    const unsigned to = this->dst(lds_tile);
    if (__builtin_expect(this->plain(row0, 32, N), 1)) {
      const char* b = this->slice + row0 * this->snb;
#pragma unroll
      for (int i = 0; i < this->PPW; ++i) copy_piece(i < 4 ? b : b + 16 * this->snb, this->off[i & 3], to + i * 1024);
      return;
    }
    int ln = threadIdx.x;
    asm volatile("" : "+v"(ln));              // (nothing of this path is worth a register outside of it)
    ln &= 63;
#pragma unroll 1
    for (int i = 0; i < this->PPW; ++i) {
      const int r = 4 * (this->PPW * this->w + i) + (ln >> 4);
      if (ZEROS && row0 + r >= N)
        *(__attribute__((address_space(3))) v4i*)(uintptr_t)(to + i * 1024 + ln * 16) = v4i{};
      else
        copy_piece(this->slice + min(row0 + r, N - 1) * this->snb + (((ln & 15) ^ swz(r)) << 4), to + i * 1024);
    }
  }
};

__device__ __forceinline__ int xattn_len(const XattnArgs& a, int b) {
  return a.lens ? min(max(__builtin_amdgcn_readfirstlane(a.lens[b]), 0), a.Nk) : a.Nk;
}

// Query row r of a key head (head after head): its place in a tensor laid out by L.
struct QueryRows {
  long long base, sh, sn;
  int Nq;
  __device__ __forceinline__ QueryRows(const XattnArgs& a, const Layout& L, int b, int g)
      : base(b * L.sb + (long long)g * a.group * L.sh), sh(L.sh), sn(L.sn), Nq(a.Nq) {}
  __device__ __forceinline__ long long at(int r) const {
    const int head = (unsigned)r / (unsigned)Nq;
    return base + head * sh + (long long)(r - head * Nq) * sn;
  }
};
// The 32 rows of a wavefront as operands; rows that do not exist are zeros.
__device__ __forceinline__ void query_operands(const bf16_t* x, const QueryRows& at, int r, int rows, int hf, uint4 (&f)[8]) {
  const bf16_t* p = x + at.at(min(r, rows - 1));
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) f[ks] = r < rows ? *(const uint4*)(p + 16 * ks + 8 * hf) : uint4{0u, 0u, 0u, 0u};
}
// A wavefront's 32 rows x 128 channels (lane = row, registers = channels) out: in whole rows where they lie in one head, as
// store_rows; else row by row.
__device__ __forceinline__ void store_query_rows(unsigned char* lds, const v16f (&x)[4], int lane, bf16_t* to, const QueryRows& at, int r0, int rows) {
  if (r0 >= rows) return;
  const int last = min(r0 + 31, rows - 1);
  if ((unsigned)r0 / (unsigned)at.Nq == (unsigned)last / (unsigned)at.Nq) {
    store_rows(lds, x, lane, to + at.at(r0), at.sn, last - r0 + 1);
    return;
  }
  const int r = r0 + (lane & 31), hf = lane >> 5;
  if (r < rows) {
    bf16_t* p = to + at.at(r) + 4 * hf;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(uint2*)(p + 32 * ct + 8 * g) = uint2{pack_bf16x2(x[ct][4 * g], x[ct][4 * g + 1]), pack_bf16x2(x[ct][4 * g + 2], x[ct][4 * g + 3])};
  }
}
// The same as fp32 rows of a partial result.
__device__ __forceinline__ void store_partial(float* row, const v16f (&x)[4], int hf) {
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(float4*)(row + 32 * ct + 8 * g + 4 * hf) = float4{x[ct][4 * g], x[ct][4 * g + 1], x[ct][4 * g + 2], x[ct][4 * g + 3]};
}

// s plus both halves of a word of bf16 numbers.
__device__ __forceinline__ float bf16_pair_sum(uint32_t w, float s) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, w), __builtin_bit_cast(v2bf, 0x3F803F80u), s, false);
}

// LSE: the log-sum-exp is wanted too (of the unrounded weights: its own sum).  SPLIT: a piece of the walk, to the workspace.
//
// A step is 32 keys: 8 KiB each of K and V in one half of a ring of two.  Kept to 168 registers and 32 KiB, so that three wavefronts
// share a SIMD: one issues products, one its exponentials, one waits for its queries or for its rows to leave.  With 64 keys a step
// (224 registers, 64 KiB, two wavefronts): 12 x 32760 queries to 64 keys 39.0 us, now 37.7, to 512 116 / 106, to 8192 1447 / 1405; 40 x
// 75600 to 512 911 / 842 (side by side on one card; 823 to 944 over cards, by the clock that power leaves them).
// For that the operands come in one stream of LDS reads, three ahead of their products (K as rows, then V transposed), the weights
// are summed on the vector ALU (a product with ones took 16 registers and one in nine of the matrix instructions), and whole walks
// take two steps a turn, so that the halves of the ring are constants and the addresses of the reads are formed once; the last
// steps, where a key may not exist, and pieces of a walk go through a body of their own.
template <int NW, bool LSE, bool SPLIT>
__global__ void __launch_bounds__(NW * 64, NW == 4 ? 3 : 2) xattn_fwd_kernel(XattnArgs a) {
  constexpr int DEEP = 3, STEP = 32, STEP_B = 2 * SWZ_TILE_B;
  __shared__ __attribute__((aligned(16))) unsigned char ring[2 * STEP_B];   // two steps' tiles, of K, then of V
  unsigned unit;
  if (!xattn_unit((unsigned)a.G * a.fwd.splits * a.fwd.tiles, a.B, unit)) return;
  const int rest = unit / (unsigned)a.fwd.tiles, tile = unit - (unsigned)rest * a.fwd.tiles;
  const int split = SPLIT ? (unsigned)rest % (unsigned)a.fwd.splits : 0, bg = SPLIT ? (unsigned)rest / (unsigned)a.fwd.splits : rest;
  const int b = (unsigned)bg / (unsigned)a.G, g = bg - b * a.G;
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), l32 = lane & 31, hf = lane >> 5;
  const int len = xattn_len(a, b), k0 = SPLIT ? split * a.fwd.chunk : 0, k1 = SPLIT ? min(len, k0 + a.fwd.chunk) : len;
  const int r0 = (tile * NW + w) * 32;
  uint4 qf[8];
  query_operands(a.q, QueryRows(a, a.lq, b, g), r0 + l32, a.rows, hf, qf);
  v16f o[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) o[ct] = v16f{};
  float m = -FLT_MAX, l = 0.f, lx = 0.f;       // l: the running sum of the rounded weights of this lane's keys
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)ring;
  if (k0 < k1) {
    AlignedCopy<NW> ck, cv;
    ck.init(a.k + b * a.lk.sb + g * a.lk.sh, a.lk.sn, w, lane);
    cv.init(a.v + b * a.lv.sb + g * a.lv.sh, a.lv.sn, w, lane);
    const int n_off = swz_lane_offset(l32, hf), t_off = swz_tr_lane_offset(lane);
    auto request = [&](int key0, int half) __attribute__((always_inline)) {
      ck.tile(key0, len, lds0 + half * STEP_B);
      cv.template tile<true>(key0, len, lds0 + half * STEP_B + SWZ_TILE_B);   // (zero times what lies behind the last key need not be zero)
    };
    request(k0, 0);
    // `half`: of the ring, a constant or not; whole: every key of the step exists
    auto step = [&](int key0, auto half, auto whole) __attribute__((always_inline)) {
      constexpr bool FIXED = !std::is_same<decltype(half), int>::value;
      copies_barrier<0>();                     // this step's tiles have landed; those of the step before are consumed
      if (key0 + STEP < k1) request(key0 + STEP, half ^ 1);
      const unsigned char* mine = ring + (FIXED ? half * STEP_B : 0);
      int no = n_off + (FIXED ? 0 : half * STEP_B), to = t_off + (FIXED ? 0 : half * STEP_B);
      if constexpr (!FIXED) asm volatile("" : "+v"(no), "+v"(to));
      auto operand = [&](int i) __attribute__((always_inline)) {
        return i < 8 ? n_op_swz(mine, no, i) : t_op_swz(mine + SWZ_TILE_B, to, i & 3, (i - 8) >> 2);
      };
      uint4 op[DEEP];
#pragma unroll
      for (int i = 0; i < DEEP; ++i) op[i] = operand(i);
      __builtin_amdgcn_sched_barrier(0);
      v16f s = v16f{};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s = mfma_bf16(op[i % DEEP], qf[i], s);
        op[i % DEEP] = operand(i + DEEP);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (!decltype(whole)::value) {
        const int left = k1 - key0 - 4 * hf;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) >= left) s[r] = -INFINITY;
      }
      float mx = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
      // The reference m moves only when the step's maximum exceeds it by more than 2^8: the weights then stay below 2^8
      // (harmless in bf16 and fp32) and the accumulators are rescaled a few times per row instead of every step.
      if (__any(mx * a.c2 > m + 8.0f)) {
        mx = fmaxf(mx, partner_f32(mx)) * a.c2;
        const float m_new = mx > m + 8.0f ? mx : m;
        const float alpha = __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= alpha;
        if constexpr (LSE) lx *= alpha;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[ct][r] *= alpha;
      }
      auto weight = [&](int r) __attribute__((always_inline)) {
        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c2, -m));
        if constexpr (LSE) lx += s[r];
      };
#pragma unroll
      for (int r = 0; r < 8; ++r) weight(r);
#pragma unroll
      for (int u = 0; u < 2; ++u) {            // 16 keys; behind the first ones' products the others' exponentials
        const uint4 pb = acc_operand(s, u);
        l = bf16_pair_sum(pb.w, bf16_pair_sum(pb.z, bf16_pair_sum(pb.y, bf16_pair_sum(pb.x, l))));
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) {
          const int i = 8 + 4 * u + ct;
          o[ct] = mfma_bf16(op[i % DEEP], pb, o[ct]);
          if (i + DEEP < 16) op[i % DEEP] = operand(i + DEEP);
          if (u == 0) {
            weight(8 + 2 * ct);
            weight(9 + 2 * ct);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    int key0 = k0;
    if constexpr (!SPLIT) {
      for (; key0 + 2 * STEP <= k1; key0 += 2 * STEP) {
        step(key0, std::integral_constant<int, 0>{}, std::true_type{});
        step(key0 + STEP, std::integral_constant<int, 1>{}, std::true_type{});
      }
    }
#pragma unroll 1
    for (int half = 0; key0 < k1; key0 += STEP, half ^= 1) step(key0, half, std::false_type{});
  }
  // (formed again: not worth registers through the walk)
  int th = threadIdx.x;
  asm volatile("" : "+v"(th));
  const int ln = th & 63, upper = ln >> 5, row = r0 + (ln & 31);
  l += partner_f32(l);                         // (0: no key)
  if constexpr (LSE) lx += partner_f32(lx);
  const long long first = ((long long)b * a.H + g * a.group) * a.Nq;   // of this key head's query rows among all
  if constexpr (SPLIT) {
    if (row < a.rows) {
      const long long at = (long long)split * a.B * a.H * a.Nq + first + row;
      if (upper == 0) *(float4*)(a.part_ml + 4 * at) = float4{m, l, LSE ? lx : l, 0.f};
      store_partial(a.part_o + at * D, o, upper);
    }
  } else {
    const float inv = l > 0.f ? 1.0f / l : 0.f;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[ct][r] *= inv;
    if constexpr (LSE) {
      if (upper == 0 && row < a.rows) a.lse[first + row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(lx)) * LN2;   // (a NaN is not "no key")
    }
    copies_barrier<0>();                       // nobody reads the last step's tiles any more
    store_query_rows(ring + w * 8192, o, ln, a.out, QueryRows(a, a.lo, b, g), r0, a.rows);
  }
}

// One row per workgroup (or eight, half a wavefront each, where there are few pieces: !WIDE).  The pieces' maxima and sums are
// read side by side, a lane each, and leave their weights 2^(m - max m) in LDS; then the pieces' rows are added up, dealt to
// the eight halves of wavefronts (WIDE).  With the maxima read one after the other by every thread, 118 pieces took 28 us.
template <bool WIDE>
__global__ void __launch_bounds__(256) xattn_join_kernel(XattnArgs a) {
  __shared__ float weight[WIDE ? XATTN_PIECES : 1];
  __shared__ float4 red_o[8][32];
  __shared__ float red[3][4];
  const int t = threadIdx.x, half = t >> 5, c = t & 31, lane = t & 63;
  const long long all = (long long)a.B * a.H * a.Nq, row = WIDE ? blockIdx.x : min(8ll * blockIdx.x + half, all - 1);
  const int S = a.fwd.splits;
  float M = -FLT_MAX, l = 0.f, lx = 0.f;
  float4 o{0.f, 0.f, 0.f, 0.f};
  auto piece = [&](int s, float w) __attribute__((always_inline)) {
    // (a piece without keys has weight 0, and its row may hold anything finite: it was written as zeros)
    const float4 p = *(const float4*)(a.part_o + (s * all + row) * D + 4 * c);
    o.x = __builtin_fmaf(w, p.x, o.x); o.y = __builtin_fmaf(w, p.y, o.y);
    o.z = __builtin_fmaf(w, p.z, o.z); o.w = __builtin_fmaf(w, p.w, o.w);
  };
  if constexpr (WIDE) {
    float4 ml[XATTN_PIECES / 256];
#pragma unroll
    for (int u = 0; u < XATTN_PIECES / 256; ++u) {
      const int s = t + 256 * u;
      ml[u] = float4{-FLT_MAX, 0.f, 0.f, 0.f};
      if (s < S) ml[u] = *(const float4*)(a.part_ml + 4 * (s * all + row));
      M = fmaxf(M, ml[u].x);
    }
    M = rows_max(row_max(M));
    if (lane == 0) red[0][t >> 6] = M;
    __syncthreads();
    M = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
#pragma unroll
    for (int u = 0; u < XATTN_PIECES / 256; ++u) {
      const float w = __builtin_amdgcn_exp2f(ml[u].x - M);
      if (t + 256 * u < S) weight[t + 256 * u] = w;
      l = __builtin_fmaf(w, ml[u].y, l);
      lx = __builtin_fmaf(w, ml[u].z, lx);
    }
    l = rows_sum(row_sum(l));
    lx = rows_sum(row_sum(lx));
    if (lane == 0) { red[1][t >> 6] = l; red[2][t >> 6] = lx; }
    __syncthreads();
    l = red[1][0] + red[1][1] + red[1][2] + red[1][3];
    lx = red[2][0] + red[2][1] + red[2][2] + red[2][3];
#pragma unroll 4
    for (int s = half; s < S; s += 8) piece(s, weight[s]);
    red_o[half][c] = o;
    __syncthreads();
    if (half != 0) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      const float4 p = red_o[i][c];
      o.x += p.x; o.y += p.y; o.z += p.z; o.w += p.w;
    }
  } else {
    float4 ml[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      ml[s] = *(const float4*)(a.part_ml + 4 * (min(s, S - 1) * all + row));
      M = fmaxf(M, ml[s].x);
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const float w = s < S ? __builtin_amdgcn_exp2f(ml[s].x - M) : 0.f;
      l = __builtin_fmaf(w, ml[s].y, l);
      lx = __builtin_fmaf(w, ml[s].z, lx);
      if (s < S) piece(s, w);
    }
    if (8ll * blockIdx.x + half >= all) return;
  }
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  const long long bh = row / a.Nq;
  const int n = (int)(row - bh * a.Nq), b = (int)(bh / a.H), h = (int)(bh - (long long)b * a.H);
  *(uint2*)(a.out + b * a.lo.sb + h * a.lo.sh + n * a.lo.sn + 4 * c) = uint2{pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv)};
  if (a.lse && c == 0) a.lse[row] = l == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(lx)) * LN2;
}

// ---------------------------------------------------------------------------
// dS = P o (dO V^T - delta) with P = 2^(S - lse), dQ = scale dS K: three products of a tile pair, S and dP formed again rather than
// kept (a matrix of 400 MB at 12 x 32760 x 512).  P and dS are fp32 until dS is rounded to the bf16 operand of the last product.
// delta takes the forward pass's bf16 out: an error of up to 2^-8 |dout| . |out| in it, which is 1.0e-3 of dQ and dK in norm beside 1.7e-3
// each for dS as a bf16 operand and for the result's own rounding; a sum of P dP in fp32 would take another walk over the keys.
// Two wavefronts per SIMD (q, dO and dQ alone are 128 registers); 12 x 32760 queries to 512 keys 182 us (0.85 PFLOP/s, 400 MB), at
// longer walks 1.2 PFLOP/s: power.  Operands read four products ahead in a fixed order: 181.
template <int NW, bool SPLIT>
__global__ void __launch_bounds__(NW * 64, 2) xattn_dq_kernel(XattnArgs a) {
  constexpr int KT = NW == 4 ? 2 : 1, STEP_B = 2 * KT * SWZ_TILE_B, STEP = 32 * KT;
  __shared__ __attribute__((aligned(16))) unsigned char ring[2 * STEP_B];
  unsigned unit;
  if (!xattn_unit((unsigned)a.G * a.dqd.splits * a.dqd.tiles, a.B, unit)) return;
  const int rest = unit / (unsigned)a.dqd.tiles, tile = unit - (unsigned)rest * a.dqd.tiles;
  const int split = SPLIT ? (unsigned)rest % (unsigned)a.dqd.splits : 0, bg = SPLIT ? (unsigned)rest / (unsigned)a.dqd.splits : rest;
  const int b = (unsigned)bg / (unsigned)a.G, g = bg - b * a.G;
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), l32 = lane & 31, hf = lane >> 5;
  const int len = xattn_len(a, b), k0 = SPLIT ? split * a.dqd.chunk : 0, k1 = SPLIT ? min(len, k0 + a.dqd.chunk) : len;
  const int r0 = (tile * NW + w) * 32, row = r0 + l32;
  v16f dq[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) dq[ct] = v16f{};
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)ring;
  if (k0 < k1) {
    uint4 qf[8], df[8];
    query_operands(a.q, QueryRows(a, a.lq, b, g), row, a.rows, hf, qf);
    query_operands(a.dout, QueryRows(a, a.ldo, b, g), row, a.rows, hf, df);
    // The row's base-2 log-sum-exp and delta = dout . out, half of its channels in each lane of the pair; for the dk, dv kernel
    // too, padded to whole steps of its walk (lse = +infinity: weights of exactly zero).
    float lse2 = INFINITY, neg_delta = 0.f;
    {
      const bf16_t* o = a.o + QueryRows(a, a.lo, b, g).at(min(row, a.rows - 1));
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        float x[8], y[8];
        unpack8(*(const uint4*)(o + 16 * ks + 8 * hf), x);
        unpack8(df[ks], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) neg_delta = __builtin_fmaf(-x[e], y[e], neg_delta);
      }
      neg_delta += partner_f32(neg_delta);
      if (row < a.rows) {
        const int head = (unsigned)row / (unsigned)a.Nq, n = row - head * a.Nq, padded = xattn_padded_rows(a.Nq);
        const long long bh = (long long)b * a.H + g * a.group + head;
        lse2 = a.lse_in[bh * a.Nq + n] * LOG2E;
        if (hf == 0 && split == 0) {
          a.lse2[bh * padded + n] = lse2;
          a.neg_delta[bh * padded + n] = neg_delta;
          if (n == a.Nq - 1)
            for (int i = n + 1; i < padded; ++i) {
              a.lse2[bh * padded + i] = INFINITY;
              a.neg_delta[bh * padded + i] = 0.f;
            }
        }
      }
    }
    AlignedCopy<NW> ck, cv;
    ck.init(a.k + b * a.lk.sb + g * a.lk.sh, a.lk.sn, w, lane);
    cv.init(a.v + b * a.lv.sb + g * a.lv.sh, a.lv.sn, w, lane);
    const int n_off = swz_lane_offset(l32, hf), t_off = swz_tr_lane_offset(lane);
    // (keys behind the last come as the last one: their weights are zero)
    auto request = [&](int key0, int half) __attribute__((always_inline)) {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        ck.tile(key0 + 32 * kt, len, lds0 + half * STEP_B + kt * SWZ_TILE_B);
        cv.tile(key0 + 32 * kt, len, lds0 + half * STEP_B + (KT + kt) * SWZ_TILE_B);
      }
    };
    request(k0, 0);
    int half = 0;
    for (int key0 = k0; key0 < k1; key0 += STEP, half ^= 1) {
      copies_barrier<0>();
      if (key0 + STEP < k1) request(key0 + STEP, half ^ 1);
      int no = n_off + half * STEP_B, to = t_off + half * STEP_B;
      asm volatile("" : "+v"(no), "+v"(to));
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const unsigned char *tk = ring + kt * SWZ_TILE_B, *tv = ring + (KT + kt) * SWZ_TILE_B;
        v16f s = v16f{}, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = neg_delta;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          s = mfma_bf16(n_op_swz(tk, no, ks), qf[ks], s);
          dp = mfma_bf16(n_op_swz(tv, no, ks), df[ks], dp);
        }
        if (key0 + 32 * kt + 32 > k1) {
          const int left = k1 - key0 - 32 * kt - 4 * hf;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (8 * (r >> 2) + (r & 3) >= left) s[r] = -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c2, -lse2)) * dp[r];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint4 ds = acc_operand(s, u);
#pragma unroll
          for (int ct = 0; ct < 4; ++ct) dq[ct] = mfma_bf16(t_op_swz(tk, to, ct, u), ds, dq[ct]);
        }
      }
    }
  }
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[ct][r] *= a.scale;
  if constexpr (SPLIT) {
    if (row < a.rows)
      store_partial(a.part_dq + ((long long)split * a.B * a.H * a.Nq + ((long long)b * a.H + g * a.group) * a.Nq + row) * D, dq, hf);
  } else {
    copies_barrier<0>();
    store_query_rows(ring + w * 8192, dq, lane, a.dq, QueryRows(a, a.ldq, b, g), r0, a.rows);
  }
}

// dV = P^T dO, dK = scale dS^T Q.  A wavefront owns 32 keys and walks over the query rows of every head of its group, 32 QT rows
// a step; P and dS are rounded to bf16 as operands, the sums stay in fp32 in registers (and in the workspace, where a walk is split:
// few key blocks have to fill the chip, and their pieces are added up in a fixed order).  12 x 32760 queries to 512 keys, ten pieces: 205
// us, 1.0 PFLOP/s, the matrix pipe 49 % busy at 1.93 GHz: neither it nor power (which leaves 1.5 GHz) binds, but the order of LDS
// reads, exponentials and products in two wavefronts per SIMD.  With one wavefront per SIMD and the compiler's order 348.
template <int NW, bool SPLIT>
__global__ void __launch_bounds__(NW * 64, NW == 4 ? 2 : 1) xattn_dkv_kernel(XattnArgs a) {
  constexpr int QT = 2, STEP_B = 2 * QT * SWZ_TILE_B + 512, STEP = 32 * QT, DEEP = 2;  // Q, dO, then lse2 and -delta of the rows
  __shared__ __attribute__((aligned(16))) unsigned char ring[2 * STEP_B];
  unsigned unit;
  if (!xattn_unit((unsigned)a.G * a.dkv.splits * a.dkv.tiles, a.B, unit)) return;
  const int rest = unit / (unsigned)a.dkv.tiles, tile = unit - (unsigned)rest * a.dkv.tiles;
  const int split = SPLIT ? (unsigned)rest % (unsigned)a.dkv.splits : 0, bg = SPLIT ? (unsigned)rest / (unsigned)a.dkv.splits : rest;
  const int b = (unsigned)bg / (unsigned)a.G, g = bg - b * a.G;
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), l32 = lane & 31, hf = lane >> 5;
  const int len = xattn_len(a, b), key0 = (tile * NW + w) * 32, key = key0 + l32;
  const int per_head = (a.Nq + STEP - 1) / STEP, total = a.group * per_head;
  const int s0 = SPLIT ? split * a.dkv.chunk : 0, s1 = SPLIT ? min(total, s0 + a.dkv.chunk) : total;
  v16f dk[4], dv[4];
#pragma unroll
  for (int ct = 0; ct < 4; ++ct) dk[ct] = dv[ct] = v16f{};
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)ring;
  if (tile * NW * 32 < len && s0 < s1) {       // (uniform)
    uint4 kf[8], vf[8];
    own_rows(a.k + b * a.lk.sb + g * a.lk.sh, a.lk.sn, key, len, hf, kf);
    own_rows(a.v + b * a.lv.sb + g * a.lv.sh, a.lv.sn, key, len, hf, vf);
    AlignedCopy<NW> cq, cd;
    const bf16_t *q0 = a.q + b * a.lq.sb + (long long)g * a.group * a.lq.sh, *d0 = a.dout + b * a.ldo.sb + (long long)g * a.group * a.ldo.sh;
    cq.init(q0, a.lq.sn, w, lane);
    cd.init(d0, a.ldo.sn, w, lane);
    const long long stat0 = ((long long)b * a.H + g * a.group) * xattn_padded_rows(a.Nq);
    const int n_off = swz_lane_offset(l32, hf), t_off = swz_tr_lane_offset(lane);
    int head = (unsigned)s0 / (unsigned)per_head, in_head = s0 - head * per_head;   // of the step requested next
    auto request = [&](int half) __attribute__((always_inline)) {
      cq.slice = (const char*)(q0 + head * a.lq.sh);
      cd.slice = (const char*)(d0 + head * a.ldo.sh);
      const int row0 = in_head * STEP;
#pragma unroll
      for (int x = 0; x < QT; ++x) {           // (rows behind a head's last come as its last: their weights are zero)
        cq.tile(row0 + 32 * x, a.Nq, lds0 + half * STEP_B + x * SWZ_TILE_B);
        cd.tile(row0 + 32 * x, a.Nq, lds0 + half * STEP_B + (QT + x) * SWZ_TILE_B);
      }
      if (w == 0) {
        const long long at = stat0 + (long long)head * xattn_padded_rows(a.Nq) + row0;
        copy_floats(a.lse2 + at, 4u * lane, lds0 + half * STEP_B + 2 * QT * SWZ_TILE_B);
        copy_floats(a.neg_delta + at, 4u * lane, lds0 + half * STEP_B + 2 * QT * SWZ_TILE_B + 256);
      }
      if (++in_head == per_head) {
        in_head = 0;
        ++head;
      }
    };
    request(0);
    int half = 0;
    for (int step = s0; step < s1; ++step, half ^= 1) {
      copies_barrier<0>();
      if (step + 1 < s1) request(half ^ 1);
      int no = n_off + half * STEP_B, to = t_off + half * STEP_B;
      asm volatile("" : "+v"(no), "+v"(to));
      const unsigned char* stat = ring + half * STEP_B + 2 * QT * SWZ_TILE_B + 16 * hf;
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        // The tile's 32 products take their operands from one stream of LDS reads, two ahead: Q and dO as rows (S, dP), then
        // both transposed (dV, dK in turn).  Held to that order, the sums, the keys' operands and what is in flight fit 256
        // registers: two wavefronts share a SIMD.
        const unsigned char *tq = ring + x * SWZ_TILE_B, *td = ring + (QT + x) * SWZ_TILE_B;
        auto flip = [](int off, int bits) __attribute__((always_inline)) {   // (formed anew each time: sixteen addresses held would not fit)
          int a;
          asm volatile("v_xor_b32 %0, %2, %1" : "=v"(a) : "v"(off), "n"(bits));
          return a;
        };
        auto operand = [&](int i) __attribute__((always_inline)) {
          if (i < 16) return *(const uint4*)((i < 8 ? tq : td) + flip(no, (i & 7) << 5));
          const int u = (i - 16) >> 3, ct = ((i - 16) >> 1) & 3;
          const unsigned char* tile = (i & 1) ? tq : td;
          union { v4s h[2]; uint4 v; } r;
          r.h[0] = read_tr(tile + 16 * u * 256 + flip(to, ct << 6));
          r.h[1] = read_tr(tile + (16 * u + 8) * 256 + flip(to, (ct << 6) ^ (2 << 4)));
          return r.v;
        };
        uint4 op[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) op[i] = operand(i);
        v16f s = v16f{}, dp;
#pragma unroll
        for (int u = 0; u < 4; ++u) {          // (rows 8 u + 4 hf + 0..3 of the tile)
          const float4 d4 = *(const float4*)(stat + 256 + 128 * x + 32 * u);
          dp[4 * u] = d4.x; dp[4 * u + 1] = d4.y; dp[4 * u + 2] = d4.z; dp[4 * u + 3] = d4.w;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s = mfma_bf16(op[i % DEEP], kf[i], s);
          op[i % DEEP] = operand(i + DEEP);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 8; i < 16; ++i) {         // behind a product: two exponentials
          dp = mfma_bf16(op[i % DEEP], vf[i - 8], dp);
          op[i % DEEP] = operand(i + DEEP);
          const int e = 2 * (i - 8);
          const float2 l2 = *(const float2*)(stat + 128 * x + 32 * (e >> 2) + 4 * (e & 3));
          s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c2, -l2.x));
          s[e + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], a.c2, -l2.y));
          __builtin_amdgcn_sched_barrier(0);
        }
        uint4 pb[2], db[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          pb[u] = acc_operand(s, u);
#pragma unroll
          for (int r = 8 * u; r < 8 * u + 8; ++r) dp[r] *= s[r];
          db[u] = acc_operand(dp, u);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 16; i < 32; ++i) {
          const int u = (i - 16) >> 3, ct = ((i - 16) >> 1) & 3;
          if (i & 1) dk[ct] = mfma_bf16(op[i % DEEP], db[u], dk[ct]);
          else dv[ct] = mfma_bf16(op[i % DEEP], pb[u], dv[ct]);
          if (i + DEEP < 32) op[i % DEEP] = operand(i + DEEP);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  const float keep = key < len ? a.scale : 0.f;
#pragma unroll
  for (int ct = 0; ct < 4; ++ct)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dk[ct][r] = key < len ? dk[ct][r] * keep : 0.f;      // (a key that does not exist took whatever weights zeros give)
      dv[ct][r] = key < len ? dv[ct][r] : 0.f;
    }
  if constexpr (SPLIT) {
    if (key < a.Nk) {
      const long long at = (((long long)split * a.B + b) * a.G + g) * a.Nk + key;
      store_partial(a.part_dk + at * D, dk, hf);
      store_partial(a.part_dv + at * D, dv, hf);
    }
  } else {
    copies_barrier<0>();
    if (key0 < a.Nk) {
      unsigned char* mine = ring + w * 8192;
      store_rows(mine, dk, lane, a.dk + b * a.ldk.sb + g * a.ldk.sh + key0 * a.ldk.sn, a.ldk.sn, a.Nk - key0);
      store_rows(mine, dv, lane, a.dv + b * a.ldv.sb + g * a.ldv.sh + key0 * a.ldv.sn, a.ldv.sn, a.Nk - key0);
    }
  }
}

// to[b][h][n] = sum over s of part[s][b][h][n], in the order of s, eight rows per workgroup; blockIdx.y: which of two tensors.
struct XattnSum {
  const float* part[2];
  bf16_t* to[2];
  Layout L[2];
  int splits, H, N;
  long long rows;
};
__global__ void __launch_bounds__(256) xattn_sum_kernel(XattnSum x) {
  const int c = threadIdx.x & 31, y = blockIdx.y;
  const long long row = 8ll * blockIdx.x + (threadIdx.x >> 5);
  if (row >= x.rows) return;
  float4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < x.splits; ++s) {
    const float4 p = *(const float4*)(x.part[y] + (s * x.rows + row) * D + 4 * c);
    o.x += p.x; o.y += p.y; o.z += p.z; o.w += p.w;
  }
  const long long bh = row / x.N;
  const int n = (int)(row - bh * x.N), b = (int)(bh / x.H), h = (int)(bh - (long long)b * x.H);
  *(uint2*)(x.to[y] + b * x.L[y].sb + h * x.L[y].sh + n * x.L[y].sn + 4 * c) = uint2{pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w)};
}

// ---------------------------------------------------------------------------
// A walk of `steps` steps by each of `units` workgroups: in how many pieces.  A piece shortens the walk and adds its partial results
// to what is written and read back (bytes_per_piece at 5 TB/s), and splitting at all adds the launch that joins them and what a piece
// starts and ends with.  A step takes the longer the more workgroups share a compute unit.  So with c of them to a unit the time is
//   us_per_step(c) * steps / S + us_to_split + S * bytes_per_piece / 5 TB/s,   least at S = sqrt(steps us_per_step(c) / (us of a piece)),
// of what c to a unit leave room for; one piece if no c makes it less.  Measured (us, in a captured graph): 1 row of 12 heads to 512
// keys in one piece 12.7, in eight 8.9; to 2048 in 8 pieces 13.7, in 32 8.1; 256 of 12 to 4096 in one 74, in 8 25.7, in 16 26.6; 1024 of
// 12 to 512 in one 13.4, in two 21.8, to 4096 75 / 60.8, in five 46.2; 2048 of 12 to 2048 in one 41.2, in two 51.9, in four 48.8, to 8192
// 148 / 145 / 126; 4096 of 12 to 4096 113 / 128.  (With one us_per_step for every c, and 4 us to split, the rule took two pieces for
// 2048 of 12 to 2048, 512 of 40 to 2048, where one takes 41.2 and two 49.0, and 4096 of 12 to 4096.)
struct XattnCost {
  int most;                 // workgroups to a compute unit
  double us_per_step[4];    // with 1 to `most` of them
  double us_to_split;
};
static XattnDeal deal(long long units, int nw, int tiles, int walk, int step, const XattnCost& cost, double bytes_per_piece) {
  const int steps = (walk + step - 1) / step;
  const long long places = compute_units();
  const double per_piece = bytes_per_piece / 5e6;
  long long pieces = 1;
  double least = steps * cost.us_per_step[std::min<long long>((units + places - 1) / places, cost.most) - 1];
  for (int c = 1; c <= cost.most; ++c) {
    const double whole = steps * cost.us_per_step[c - 1];
    const long long p = std::min({(long long)std::sqrt(whole / per_piece), c * places / units, (long long)(steps + 1) / 2 /* two steps at least */,
                                  (long long)XATTN_PIECES});
    const double us = p < 2 ? least : whole / p + cost.us_to_split + p * per_piece;
    if (us < least) {
      least = us;
      pieces = p;
    }
  }
  const int each = (int)((steps + pieces - 1) / pieces);
  return XattnDeal{nw, tiles, (steps + each - 1) / each, each * step};
}
XattnDeal xattn_deal_rows(int B, int G, int rows, int Nk, bool fwd) {
  const int nw = rows <= 32 ? 1 : rows <= 64 ? 2 : 4, tiles = (rows + 32 * nw - 1) / (32 * nw), wide = nw == 4;
  static constexpr XattnCost few_rows{4, {0.7, 0.7, 0.7, 0.7}, 4.0}, forward{3, {0.58, 0.87, 1.4}, 10.0}, dq{2, {1.6, 1.6}, 4.0};
  return deal((long long)B * G * tiles, nw, tiles, Nk, fwd || !wide ? 32 : 64, !wide ? few_rows : fwd ? forward : dq,
              (double)B * G * rows * 2 * (D + 4) * 4);
}
XattnDeal xattn_deal_keys(int B, int G, int group, int Nq, int Nk) {
  const int nw = Nk <= 32 ? 1 : Nk <= 64 ? 2 : 4, tiles = (Nk + 32 * nw - 1) / (32 * nw);
  static constexpr XattnCost dkv{2, {2.0, 2.0}, 4.0};
  return deal((long long)B * G * tiles, nw, tiles, group * ((Nq + 63) / 64), 1, dkv, (double)B * G * Nk * 4 * D * 4);
}

void launch_xattn_fwd(const XattnArgs& a, hipStream_t stream) {
  const unsigned grid = xattn_numbers((unsigned)a.G * a.fwd.splits * a.fwd.tiles, a.B);
#define XATTN_FWD(NW)                                                                                                          \
  do {                                                                                                                         \
    if (a.fwd.splits > 1) {                                                                                                    \
      if (a.lse) xattn_fwd_kernel<NW, true, true><<<grid, NW * 64, 0, stream>>>(a);                               \
      else xattn_fwd_kernel<NW, false, true><<<grid, NW * 64, 0, stream>>>(a);                                    \
    } else {                                                                                                                   \
      if (a.lse) xattn_fwd_kernel<NW, true, false><<<grid, NW * 64, 0, stream>>>(a);                              \
      else xattn_fwd_kernel<NW, false, false><<<grid, NW * 64, 0, stream>>>(a);                                   \
    }                                                                                                                          \
  } while (0)
  if (a.fwd.nw == 1) XATTN_FWD(1);
  else if (a.fwd.nw == 2) XATTN_FWD(2);
  else XATTN_FWD(4);
#undef XATTN_FWD
  if (a.fwd.splits > 1) {
    const long long all = (long long)a.B * a.H * a.Nq;
    if (a.fwd.splits > 8) xattn_join_kernel<true><<<(unsigned)all, 256, 0, stream>>>(a);
    else xattn_join_kernel<false><<<(unsigned)((all + 7) / 8), 256, 0, stream>>>(a);
  }
}

void launch_xattn_bwd(const XattnArgs& a, hipStream_t stream) {
  const long long all = (long long)a.B * a.H * a.Nq;
  const unsigned gq = xattn_numbers((unsigned)a.G * a.dqd.splits * a.dqd.tiles, a.B), gk = xattn_numbers((unsigned)a.G * a.dkv.splits * a.dkv.tiles, a.B);
#define XATTN_BWD(KERNEL, NW, SPLIT, GRID)                                    \
  do {                                                                        \
    if (SPLIT) KERNEL<NW, true><<<GRID, NW * 64, 0, stream>>>(a);             \
    else KERNEL<NW, false><<<GRID, NW * 64, 0, stream>>>(a);                  \
  } while (0)
  const bool sq = a.dqd.splits > 1, sk = a.dkv.splits > 1;
  if (a.dqd.nw == 1) XATTN_BWD(xattn_dq_kernel, 1, sq, gq);
  else if (a.dqd.nw == 2) XATTN_BWD(xattn_dq_kernel, 2, sq, gq);
  else XATTN_BWD(xattn_dq_kernel, 4, sq, gq);
  if (a.dkv.nw == 1) XATTN_BWD(xattn_dkv_kernel, 1, sk, gk);
  else if (a.dkv.nw == 2) XATTN_BWD(xattn_dkv_kernel, 2, sk, gk);
  else XATTN_BWD(xattn_dkv_kernel, 4, sk, gk);
#undef XATTN_BWD
  if (sq) {
    const XattnSum x{{a.part_dq, nullptr}, {a.dq, nullptr}, {a.ldq, a.ldq}, a.dqd.splits, a.H, a.Nq, all};
    xattn_sum_kernel<<<dim3((unsigned)((all + 7) / 8), 1), 256, 0, stream>>>(x);
  }
  if (sk) {
    const long long keys = (long long)a.B * a.G * a.Nk;
    const XattnSum x{{a.part_dk, a.part_dv}, {a.dk, a.dv}, {a.ldk, a.ldv}, a.dkv.splits, a.G, a.Nk, keys};
    xattn_sum_kernel<<<dim3((unsigned)((keys + 7) / 8), 2), 256, 0, stream>>>(x);
  }
}

}  // namespace sla
