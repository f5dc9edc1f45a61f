// Microscaled 4-bit floating point (include/mxfp4.h): quantisation, its inverse, plain rows from and into the operand order
// (mxfp4.h), and the product of two quantised matrices.
#include "mxfp4.h"
#include "rows.h"
#include "tiles.h"

namespace sla {

// ---------------------------------------------------------------------------
// A wavefront takes a step (256 features) of 2 PAIRS rows, two rows at a time, eight features a lane: four lanes are a block, and two
// rows' records are a whole line.  NT: what is read or written once and exceeds the memory-side cache goes past the caches.
// Bound by HBM: 75600 x 5120 184 us, 5.3 TB/s, and back 140, 7.0; 512 x 5120 and back 8.3 us, one row and back 6.0: two launches.
template <int PAIRS, bool NT>
__global__ void __launch_bounds__(256) mxfp4_quantize_kernel(const bf16_t* __restrict__ x, int R, int K, int RP, int KB, int units,
                                                             uint8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
  const int unit = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  if (unit >= units) return;
  const int group = unit / KB, k8 = (unit - group * KB) * 32 + (lane & 31), r0 = group * 2 * PAIRS + (lane >> 5);
  uint4 v[PAIRS];
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    v[i] = uint4{0u, 0u, 0u, 0u};
    if (r0 + 2 * i < R && k8 < K / 8) v[i] = load_from<NT, uint4>(x + (long long)(r0 + 2 * i) * K + 8ll * k8);
  }
#pragma unroll
  for (int i = 0; i < PAIRS; ++i)
    if (r0 + 2 * i < R) mx_store8(v[i], r0 + 2 * i, k8, RP, codes, exps);   // (a quad is one row's)
}

// What eight codes of a block of exponent e stand for, as bf16.
__device__ __forceinline__ uint4 mx_values8(uint32_t four, uint32_t e) {
  if (e - 1u < 252u) {                        // (the scale a normal number, no value beyond bf16: exact)
    const float s = __uint_as_float(e << 23);
    return uint4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(four, s, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(four, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(four, s, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(four, s, 3))};
  }
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = (four >> (4 * i)) & 7u, sign = (four >> (4 * i + 3)) << 31;
    // twice the magnitude: 0, 1, 2, 3, 4, 6, 8, 12
    const float twice = m < 4 ? (float)m : (float)((4 + 2 * (m & 1)) << ((m >> 1) - 2));
    v[i] = e == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(__float_as_uint(ldexpf(twice, (int)e - 128)) | sign);
  }
  return pack8(v);
}
template <int PAIRS, bool NT>
__global__ void __launch_bounds__(256) mxfp4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ exps,
                                                               int R, int K, int RP, int KB, int units, bf16_t* __restrict__ x) {
  const int unit = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  if (unit >= units) return;
  const int group = unit / KB, kb = unit - group * KB, k8 = kb * 32 + (lane & 31), r0 = group * 2 * PAIRS + (lane >> 5), c = (k8 >> 2) & 7;
  uint32_t v[PAIRS], e[PAIRS];
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {           // (rows behind the last: what lies there, not stored)
    const int row = min(r0 + 2 * i, RP - 1);
    v[i] = *(const uint32_t*)(codes + mx_chunk_at(RP, row, kb, c) + 4 * (k8 & 3));
    e[i] = exps[mx_exp_at(RP, row, kb, c)];
  }
#pragma unroll
  for (int i = 0; i < PAIRS; ++i)
    if (r0 + 2 * i < R && k8 < K / 8) store_to<NT>(x + (long long)(r0 + 2 * i) * K + 8ll * k8, mx_values8(v[i], e[i]));
}

// One block of 32 features a thread, byte by byte (rows of codes may stand at any address): 13824 x 5120 into an object 94 us, 0.8 TB/s, out of it
// 30, 2.5; of a weight once.
__global__ void __launch_bounds__(256) mxfp4_pack_kernel(const uint8_t* __restrict__ from, const uint8_t* __restrict__ from_exps,
                                                         int R, int K, int RP, int KB, uint8_t* __restrict__ codes,
                                                         uint8_t* __restrict__ exps) {
  const long long n = (long long)R * KB * 8;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += 256ll * gridDim.x) {
    const int row = (int)(i / (KB * 8)), blk = (int)(i - (long long)row * (KB * 8)), have = max(0, min(16, K / 2 - 16 * blk));
    uint8_t* to = codes + mx_chunk_at(RP, row, blk >> 3, blk & 7);
    for (int b = 0; b < 16; ++b) to[b] = b < have ? from[(long long)row * (K / 2) + 16 * blk + b] : (uint8_t)0;
    exps[mx_exp_at(RP, row, blk >> 3, blk & 7)] = have ? from_exps[(long long)row * ((K + 31) / 32) + blk] : (uint8_t)1;
  }
}
__global__ void __launch_bounds__(256) mxfp4_unpack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ exps,
                                                           int R, int K, int RP, uint8_t* __restrict__ to, uint8_t* __restrict__ to_exps) {
  const int blocks = (K + 31) / 32;
  const long long n = (long long)R * blocks;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += 256ll * gridDim.x) {
    const int row = (int)(i / blocks), blk = (int)(i - (long long)row * blocks), have = min(16, K / 2 - 16 * blk);
    const uint8_t* at = codes + mx_chunk_at(RP, row, blk >> 3, blk & 7);
    if (to)
      for (int b = 0; b < have; ++b) to[(long long)row * (K / 2) + 16 * blk + b] = at[b];
    if (to_exps) to_exps[i] = exps[mx_exp_at(RP, row, blk >> 3, blk & 7)];
  }
}

// ---------------------------------------------------------------------------
// The product.  Weights are the A operand, so that a lane owns one token (a column of the accumulator) and runs of four
// consecutive outputs: registers 4 g .. 4 g + 3 are outputs 8 g + 4 hf + 0..3 of a tile of 32.
// ---------------------------------------------------------------------------
// Step KS of a record's four: 64 features of 32 outputs and 32 tokens; the exponents' words hold a byte per step.
template <int KS>
__device__ __forceinline__ v16f mfma_mx(const v4i& w, uint32_t we, const v4i& x, uint32_t xe, const v16f& c) {
  const v8i a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, KS, (int)we, KS, (int)xe);
}

// Few tokens or few outputs: workgroup tile (32 RT) tokens x (32 CT) outputs, whose KSPLIT wavefronts split the contraction and meet
// in LDS in a fixed order.  Operands go from memory straight to registers, a step ahead: nothing is shared between the wavefronts,
// there is no barrier in the loop.  Bound by latency, of the launch and of one round trip per step: 1 x 5120 -> 5120, 14 MB of weight,
// 5.0 us with the quantisation in it, 1 x 1536 -> 8960 3.7, 64 x 5120 -> 5120 7.3.
// QUANT: the tokens come as bf16, so few (MX_FEW features in all) that every workgroup quantises them by itself, into LDS, while its
// first weights are on their way: one launch instead of two.
constexpr int MX_FEW = 32768;
template <int RT, int CT, int KSPLIT, bool QUANT>
__global__ void __launch_bounds__(64 * KSPLIT) mxfp4_gemm_split_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xe,
                                                                       const uint8_t* __restrict__ w, const uint8_t* __restrict__ we,
                                                                       const bf16_t* __restrict__ bias, bf16_t* __restrict__ y, int M,
                                                                       int N, int K, int KB, int MT, int NT) {
  constexpr int PITCH = 36;  // floats per staged row of 32 outputs (16-byte rows, skewed banks)
  __shared__ __attribute__((aligned(16))) float part[KSPLIT][32 * RT][PITCH];
  static_assert(!QUANT || RT == 1, "up to 32 tokens");
  __shared__ __attribute__((aligned(16))) uint8_t few[QUANT ? MX_FEW / 2 : 16], few_exps[QUANT ? MX_FEW / 32 : 16];
  // XCD x takes a contiguous eighth of the tiles, along the smaller operand fastest: of the larger one a tile is then fetched into
  // one L2 only.
  const int per = (MT * NT + 7) >> 3, idx = __builtin_amdgcn_readfirstlane((int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3));
  if ((int)(blockIdx.x >> 3) >= per || idx >= MT * NT) return;
  const bool tokens_fastest = M <= N;
  const int major = __builtin_amdgcn_readfirstlane(idx / (tokens_fastest ? MT : NT)), minor = idx - major * (tokens_fastest ? MT : NT);
  const int nt = tokens_fastest ? major : minor, mt = tokens_fastest ? minor : major;
  const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6), l32 = lane & 31, hf = lane >> 5;
  const int RPx = mx_rows(M), RPw = mx_rows(N);
  const int kb0 = KB * wv / KSPLIT, kb1 = KB * (wv + 1) / KSPLIT;
  v16f acc[RT][CT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[r][c] = v16f{};
  // (tiles behind the last row: the last one once more, nothing of it is stored)
  auto row_of = [&](int tile, int RP) { return min(tile, RP / 32 - 1) * 32 + l32; };
  struct Step {
    v4i a[CT][4], b[RT][4];
    uint32_t ae[CT], be[RT];
  };
  auto load = [&](int kb, Step& s) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const int row = row_of(nt * CT + c, RPw);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) s.a[c][ks] = *(const v4i*)(w + mx_chunk_at(RPw, row, kb, 2 * ks + hf));
      s.ae[c] = *(const uint32_t*)(we + mx_exp_at(RPw, row, kb, hf));
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if constexpr (!QUANT) {
        const int row = row_of(mt * RT + r, RPx);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) s.b[r][ks] = *(const v4i*)(x + mx_chunk_at(RPx, row, kb, 2 * ks + hf));
        s.be[r] = *(const uint32_t*)(xe + mx_exp_at(RPx, row, kb, hf));
      }
    }
  };
  auto products = [&](int kb, Step& s) __attribute__((always_inline)) {
    if constexpr (QUANT) {               // (lanes behind the last token: the last one once more, for nobody)
      const int at = min(l32, M - 1) * KB + kb;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) s.b[0][ks] = *(const v4i*)(few + at * (MX_STEP / 2) + (2 * ks + hf) * 16);
      s.be[0] = *(const uint32_t*)(few_exps + at * 8 + 4 * hf);
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        acc[r][c] = mfma_mx<0>(s.a[c][0], s.ae[c], s.b[r][0], s.be[r], acc[r][c]);
        acc[r][c] = mfma_mx<1>(s.a[c][1], s.ae[c], s.b[r][1], s.be[r], acc[r][c]);
        acc[r][c] = mfma_mx<2>(s.a[c][2], s.ae[c], s.b[r][2], s.be[r], acc[r][c]);
        acc[r][c] = mfma_mx<3>(s.a[c][3], s.ae[c], s.b[r][3], s.be[r], acc[r][c]);
      }
  };
  Step s0, s1;
  if (kb0 < kb1) load(kb0, s0);
  if constexpr (QUANT) {
    // (KB * 32 is a multiple of the quad that holds a block)
    for (int i = t; i < M * KB * 32; i += 64 * KSPLIT) {
      const int row = i / (KB * 32), k8 = i - row * (KB * 32), c = (k8 >> 2) & 7;
      const uint4 v = k8 < K / 8 ? *(const uint4*)((const bf16_t*)x + (long long)row * K + 8 * k8) : uint4{0u, 0u, 0u, 0u};
      const uint32_t e = mx_exponent(__uint_as_float(quad_umax(__float_as_uint(mx_amax8(v)))));
      *(uint32_t*)(few + 4 * i) = mx_codes8(v, e);
      if ((k8 & 3) == 0) few_exps[(row * KB + (k8 >> 5)) * 8 + 4 * (c & 1) + (c >> 1)] = (uint8_t)e;
    }
    __syncthreads();
  }
  for (int kb = kb0; kb < kb1; kb += 2) {   // (a step ahead, the last one once more)
    load(min(kb + 1, kb1 - 1), s1);
    products(kb, s0);
    if (kb + 1 == kb1) break;
    load(min(kb + 2, kb1 - 1), s0);
    products(kb + 1, s1);
  }
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    if (c > 0) __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const v16f& f = acc[r][c];
        *(float4*)&part[wv][32 * r + l32][8 * g + 4 * hf] = make_float4(f[4 * g], f[4 * g + 1], f[4 * g + 2], f[4 * g + 3]);
      }
    __syncthreads();
    const int n0 = (nt * CT + c) * 32;
    for (int u = t; u < 32 * RT * 4; u += 64 * KSPLIT) {
      const int row = u >> 2, o = 8 * (u & 3), m = mt * 32 * RT + row;
      if (m >= M || n0 + o >= N) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = part[0][row][o + e];
#pragma unroll
      for (int p = 1; p < KSPLIT; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += part[p][row][o + e];
      if (bias) {
        float b8[8];
        unpack8(*(const uint4*)(bias + n0 + o), b8);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += b8[e];
      }
      *(uint4*)(y + (size_t)m * N + n0 + o) = pack8(v);
    }
  }
}

// ---------------------------------------------------------------------------
// Large calls: WM x WN wavefronts of RT x CT tiles of 32 tokens x 32 outputs.  Half a step (128 features) is a stage; STAGES of them are
// in LDS, copied without registers in between; a step's exponents ride with its first half, in two places of their own.
// A half's first 64 features are read while the second ones of the half before are multiplied; in the middle of a half, when all
// of its operands are in registers, the workgroup meets: behind that its stage is free for the half STAGES on, and the next half's
// has arrived.
// With one or two wavefronts a SIMD the products alone set the time, and what stands before and behind them: 512 x 5120 -> 13824 21.9 us
// with tiles of 256 x 128, without copies 18.6, without LDS reads too 17.2; 4096 x 5120 -> 5120 55 us, 3.9 PFLOP/s.
// ---------------------------------------------------------------------------
constexpr int MX_EPI_PITCH = 16;                  // bytes behind each staged output row
constexpr int MX_DEAL_MT = 64;                    // token tiles from which whole ones are dealt to the XCDs

// Pieces 2 i and 2 i + 1 of several consecutive ones (the immediate offset moves both addresses).
__device__ __forceinline__ void copy_pair(const char* base, unsigned off, unsigned lds_addr, int i) {
  if (i == 0)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0\n\tglobal_load_lds_dwordx4 %1, %0 offset:1024"
                 : : "s"(base), "v"(off), "s"(lds_addr) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0 offset:0x800\n\tglobal_load_lds_dwordx4 %1, %0 offset:0xc00"
                 : : "s"(base), "v"(off), "s"(lds_addr) : "memory", "m0");
}

// Workgroups are dealt round-robin over the 8 XCDs.  An XCD walks its tiles in patches of 8 tiles along the outputs, 4 or 8 along
// the tokens, what its 32 compute units hold at a time, so that each record of a step is fetched into its L2 once for several
// users; of many token tiles it takes every eighth, of few an eighth of all tiles.
struct MxTiles {
  int first, rows, NT, n, xcd;    // n: tiles of this XCD
  bool deal;
  __device__ __forceinline__ MxTiles(int xcd_, int MT, int NT_) : NT(NT_), xcd(xcd_), deal(MT >= MX_DEAL_MT) {
    const int share = (MT * NT + 7) >> 3;
    first = deal ? 0 : xcd * share;
    rows = deal ? (MT - xcd + 7) >> 3 : MT;
    n = deal ? rows * NT : min(share, MT * NT - first);
  }
  __device__ __forceinline__ void at(int slot, int& mt, int& nt) const {
    const int idx = first + slot, band = idx / (8 * NT), in_band = idx - band * 8 * NT, band_rows = min(8, rows - 8 * band);
    const int grp = in_band / (8 * band_rows), in_grp = in_band - grp * 8 * band_rows;
    const int cols = min(8, NT - 8 * grp), row = 8 * band + in_grp / cols;
    mt = __builtin_amdgcn_readfirstlane(deal ? 8 * row + xcd : row);
    nt = __builtin_amdgcn_readfirstlane(8 * grp + in_grp % cols);
  }
};

template <int WM, int WN, int RT, int CT, int STAGES>
struct MxTile {
  static constexpr int M = 32 * RT * WM, N = 32 * CT * WN;          // tokens and outputs
  static constexpr int XP = M / 64, WP = N / 64;                    // a wavefront's pieces (16 records, 1 KiB) of a half
  static constexpr int COPIES = (XP + WP) / 2;                      // ... two at a time
  static constexpr int EX = M / 128, EW = N / 128;                  // pieces (128 rows, 1 KiB) of a step's exponents: one a wavefront
  static constexpr int STAGE = (M + N) * MX_REC, EXPS = (M + N) * 8;
  static constexpr int LDS = STAGES * STAGE + 2 * EXPS;             // (exponents of two steps)
  static constexpr int TAIL = (STAGES + 1) / 2;                     // last steps, behind which less than the usual is copied
  static constexpr int EPI = 32 * CT * 2 + MX_EPI_PITCH;            // bytes of a staged output row
  // A wavefront's copies of halves `from` .. `to` (counted from a step's first) that are under way where `left` steps follow that one.
  static constexpr int copies(int from, int to, int left) {
    int n = 0;
    for (int h = from; h <= to; ++h) n += h / 2 <= left ? XP + WP + (h % 2 == 0) : 0;
    return n;
  }
  static_assert(WM * WN == 4 && M % 128 == 0 && N % 128 == 0 && M <= MX_TILE_ROWS && N <= MX_TILE_ROWS && EX + EW <= 4 && STAGES >= 3 && STAGES <= 4, "the copies' shares");
  static_assert(4 * 32 * EPI <= STAGES * STAGE && EPI % 16 == 0, "output staging fits the stages");
};

template <int WM, int WN, int RT, int CT, int STAGES, int PER_CU>
__global__ void __launch_bounds__(256, PER_CU) mxfp4_gemm_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xe,
                                                                 const uint8_t* __restrict__ w, const uint8_t* __restrict__ we,
                                                                 const bf16_t* __restrict__ bias, bf16_t* __restrict__ y, int M, int N,
                                                                 int KB, int MT, int NT) {
  using T = MxTile<WM, WN, RT, CT, STAGES>;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[T::LDS];
  const MxTiles tiles(blockIdx.x & 7, MT, NT);
  if ((int)(blockIdx.x >> 3) >= tiles.n) return;
  int mt, nt;
  tiles.at(blockIdx.x >> 3, mt, nt);
  const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6), l32 = lane & 31, hf = lane >> 5;
  const int wm = WN == 1 ? wv : wv / WN, wn = WN == 1 ? 0 : wv % WN;
  const int RPx = mx_rows(M), RPw = mx_rows(N);
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)lds;

  // This wavefront's copies: XP pieces of a half's tokens, WP of its weight; one of a step's exponents (wavefronts beyond their
  // number repeat the last).  (Rows behind the last: whatever lies there, see mx_object_bytes.)
  const unsigned lane16 = lane * 16;
  const int ep = min(wv, T::EX + T::EW - 1);
  const bool ex = ep < T::EX;
  const char* const px = (const char*)x + ((size_t)mt * T::M + 16 * T::XP * wv) * MX_REC;
  const char* const pw = (const char*)w + ((size_t)nt * T::N + 16 * T::WP * wv) * MX_REC;
  const char* const pe = ex ? (const char*)xe + ((size_t)mt * T::M + 128 * ep) * 8
                            : (const char*)we + ((size_t)nt * T::N + 128 * (ep - T::EX)) * 8;
  const size_t e_step = (size_t)(ex ? RPx : RPw) * 8;
  // copy i of a half's COPIES, two pieces each (one more where its step's exponents ride along)
  auto copy_one = [&](int h, int stage, int i) __attribute__((always_inline)) {
    const unsigned to = lds0 + stage * T::STAGE;
    if (i < T::XP / 2) copy_pair(px + (size_t)h * RPx * MX_REC, lane16, to + T::XP * wv * 1024, i);
    else if (i < T::COPIES) copy_pair(pw + (size_t)h * RPw * MX_REC, lane16, to + T::M * MX_REC + T::WP * wv * 1024, i - T::XP / 2);
    else copy_piece(pe + (h >> 1) * e_step, lane16, lds0 + STAGES * T::STAGE + ((h >> 1) & 1) * T::EXPS + ep * 1024);
  };
  auto copy_half = [&](int h, int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) copy_one(h, stage, i);
    if (!(h & 1)) copy_one(h, stage, T::COPIES);
  };
  const int frag = l32 * MX_REC + ((hf ^ mx_swz(l32)) << 4);
  // operand i of 64 features, in the order the products take them
  auto read_one = [&](int stage, int ks, int i, v4i (&xf)[RT], v4i (&wf)[CT]) __attribute__((always_inline)) {
    const unsigned char* s = lds + stage * T::STAGE + (frag ^ (ks << 5));
    if (i == 0) wf[0] = *(const v4i*)(s + T::M * MX_REC + CT * wn * 32 * MX_REC);
    else if (i <= RT) xf[i - 1] = *(const v4i*)(s + (RT * wm + i - 1) * 32 * MX_REC);
    else wf[i - RT] = *(const v4i*)(s + T::M * MX_REC + (CT * wn + i - RT) * 32 * MX_REC);
  };
  auto read_exp = [&](int step, int i, uint32_t (&xs)[RT], uint32_t (&ws)[CT]) __attribute__((always_inline)) {
    const unsigned char* s = lds + STAGES * T::STAGE + (step & 1) * T::EXPS + 8 * l32 + 4 * hf;
    if (i < RT) xs[i] = *(const uint32_t*)(s + (RT * wm + i) * 256);
    else ws[i - RT] = *(const uint32_t*)(s + T::M * 8 + (CT * wn + i - RT) * 256);
  };
  v16f acc[RT][CT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < CT; ++c) acc[r][c] = v16f{};

  constexpr int OPS = RT + CT, PRODUCTS = RT * CT;
  // the first halves; those under way behind the first one are few where there are few steps
#pragma unroll
  for (int h = 0; h < STAGES; ++h)
    if (h < 2 || KB > h / 2) copy_half(h, h);
  if (KB >= T::TAIL) copies_barrier<T::copies(1, STAGES - 1, T::TAIL - 1)>();
  else copies_barrier<0>();
  v4i x0[RT], w0[CT], x1[RT], w1[CT];
  uint32_t xx[RT], wx[CT], xn[RT], wn_[CT];
#pragma unroll
  for (int i = 0; i < OPS; ++i) read_one(0, 0, i, x0, w0);
#pragma unroll
  for (int i = 0; i < OPS; ++i) read_exp(0, i, xx, wx);
  int stage = 0;
// The products of 64 features, and behind each what AFTER(i) asks for: a wavefront alone on its SIMD has to keep the matrix pipe
// busy by itself.
#define MX_PRODUCTS(KS, X, W, AFTER)                                                                  \
  _Pragma("unroll") for (int i = 0; i < PRODUCTS; ++i) {                                              \
    const int c = i / RT, r = i % RT;                                                                 \
    acc[r][c] = mfma_mx<KS>(W[c], wx[c], X[r], xx[r], acc[r][c]);                                     \
    (AFTER)(i);                                                                                       \
    __builtin_amdgcn_sched_barrier(0);                                                                \
  }
// thing number i of n dealt over the products: PER behind each, from product FROM on
#define MX_DEAL(I, FROM, N, WHAT)                                                                     \
  {                                                                                                   \
    constexpr int per_ = ((N) + PRODUCTS - (FROM) - 1) / (PRODUCTS - (FROM));                         \
    _Pragma("unroll") for (int u_ = 0; u_ < per_; ++u_) {                                             \
      const int n_ = ((I) - (FROM)) * per_ + u_;                                                      \
      if ((I) >= (FROM) && n_ < (N)) { WHAT; }                                                        \
    }                                                                                                 \
  }
// (LEFT: steps behind this one, TAIL for so many or more.  A step is free of branches: the compiler would move the products past them.)
#define MX_HALF(PART, LEFT)                                                                           \
  {                                                                                                   \
    constexpr bool COPY = (PART + STAGES) / 2 <= LEFT, NEXT = LEFT > 0 || PART == 0, EXPS = LEFT > 0 && PART == 1; \
    constexpr int COPIES = COPY ? T::COPIES + ((PART + STAGES) % 2 == 0) : 0;                         \
    const int next = stage == STAGES - 1 ? 0 : stage + 1, ahead = 2 * step + PART + STAGES;           \
    _Pragma("unroll") for (int n_ = 0; n_ < 2; ++n_) read_one(stage, 1, n_, x1, w1);                  \
    MX_PRODUCTS(2 * PART, x0, w0, [&](int i) { MX_DEAL(i, 0, OPS - 2, read_one(stage, 1, n_ + 2, x1, w1)) });  \
    copies_barrier<T::copies(PART + 2, PART + STAGES - 1, LEFT)>();                                   \
    MX_PRODUCTS(2 * PART + 1, x1, w1, [&](int i) {                                                    \
      if constexpr (NEXT) MX_DEAL(i, 0, OPS, read_one(next, 0, n_, x0, w0))                           \
      if constexpr (EXPS) MX_DEAL(i, 0, OPS, read_exp(step + 1, n_, xn, wn_))                         \
      MX_DEAL(i, PRODUCTS / 4, COPIES, copy_one(ahead, stage, n_))                                    \
    });                                                                                               \
    if constexpr (EXPS) {                                                                             \
      _Pragma("unroll") for (int r = 0; r < RT; ++r) xx[r] = xn[r];                                   \
      _Pragma("unroll") for (int c = 0; c < CT; ++c) wx[c] = wn_[c];                                  \
    }                                                                                                 \
    stage = next;                                                                                     \
  }
  int step = 0;
  for (; step + T::TAIL < KB; ++step) {
    MX_HALF(0, T::TAIL)
    MX_HALF(1, T::TAIL)
  }
#define MX_LAST(LEFT)                     \
  if constexpr (LEFT < T::TAIL) {         \
    if (KB > LEFT) {                      \
      MX_HALF(0, LEFT)                    \
      MX_HALF(1, LEFT)                    \
      ++step;                             \
    }                                     \
  }
  MX_LAST(1)
  MX_LAST(0)
#undef MX_LAST
#undef MX_HALF
#undef MX_DEAL
#undef MX_PRODUCTS

  // Epilogue: bias in, bf16, through LDS so that rows leave as whole lines, past the caches.  (Behind the last meeting nobody reads
  // the stages.)
  unsigned char* my = lds + wv * (32 * T::EPI);
  const int n0 = nt * T::N + 32 * CT * wn;
  uint2 bw[CT][4];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g) bw[c][g] = make_uint2(0u, 0u);
  if (bias) {
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g) bw[c][g] = *(const uint2*)(bias + min(n0 + 32 * c + 8 * g + 4 * hf, N - 4));
  }
  constexpr int LANES = 4 * CT, ROWS = 64 / LANES;    // lanes a row of 32 CT outputs, rows an instruction
#pragma unroll
  for (int r = 0; r < RT; ++r) {
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint2 b4 = bw[c][g];
        const v16f& f = acc[r][c];
        *(uint2*)(my + l32 * T::EPI + (32 * c + 8 * g + 4 * hf) * 2) =
            make_uint2(pack_bf16x2(f[4 * g] + bf16_lo(b4.x), f[4 * g + 1] + bf16_hi(b4.x)),
                       pack_bf16x2(f[4 * g + 2] + bf16_lo(b4.y), f[4 * g + 3] + bf16_hi(b4.y)));
      }
    __builtin_amdgcn_wave_barrier();     // (a wavefront's LDS operations execute in order: only the compiler has to keep it)
#pragma unroll
    for (int it = 0; it < 32 / ROWS; ++it) {
      const int row = it * ROWS + lane / LANES, part = lane % LANES;
      const int m = mt * T::M + 32 * (RT * wm + r) + row;
      const v4i v = *(const v4i*)(my + row * T::EPI + part * 16);
      if (m < M && n0 + 8 * part < N) __builtin_nontemporal_store(v, (v4i*)(y + (size_t)m * N + n0 + part * 8));
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// The largest calls: tiles of 256 x 256, four wavefronts of 128 x 128, one per SIMD, and one workgroup per compute unit that goes
// from tile to tile.  The operands of a product then come from LDS for sixteen others instead of eight, a byte copied from L2
// serves 256 x 256 products of its feature, and nothing waits between tiles: the last half steps of one copy the first of the
// next, whose first operands are read before the results leave.  Power is what bounds this kernel: every byte that does not move
// is time.  75600 x 5120 -> 5120 868 us, 4.6 PFLOP/s, 32760 x 5120 -> 15360 1097 us, 4.7; 65520 x 1536 -> 8960 471 us, 3.8: there the results,
// 1.2 GB, leave after every six steps (413 us without their stores).  The clock is 1.72 to 1.77 GHz in it, the pipe 65 % busy;
// of 736 us at 65536 x 5120 -> 5120, 620 are left without the copies, 584 without the LDS reads, 579 for the products alone.  (K of more
// than one step.)
using MxBig = MxTile<2, 2, 4, 4, 3>;
__global__ void __launch_bounds__(256, 1) mxfp4_gemm_walk_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xe,
                                                                 const uint8_t* __restrict__ w, const uint8_t* __restrict__ we,
                                                                 const bf16_t* __restrict__ bias, bf16_t* __restrict__ y, int M, int N,
                                                                 int KB, int MT, int NT) {
  using T = MxBig;
  constexpr int RT = 4, CT = 4, OPS = RT + CT, PRODUCTS = RT * CT, STAGES = 3;
  constexpr int AT_EXPS = STAGES * T::STAGE, AT_OUT = AT_EXPS + 2 * T::EXPS, AT_BIAS = AT_OUT + 4 * 32 * T::EPI;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[AT_BIAS + 4 * 256];
  const MxTiles tiles(blockIdx.x & 7, MT, NT);
  const int walkers = gridDim.x >> 3;
  int slot = blockIdx.x >> 3;
  if (slot >= tiles.n) return;
  const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6), l32 = lane & 31, hf = lane >> 5;
  const int wm = wv >> 1, wn = wv & 1;
  const int RPx = mx_rows(M), RPw = mx_rows(N);
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
  int mt, nt, next_mt, next_nt;
  tiles.at(slot, mt, nt);

  // This wavefront's copies of a half: four pieces each of its tokens and its weight, two at a time; one of a step's exponents
  // (wavefronts 0, 1: tokens; 2, 3: weight).  px, pw, pe: where the next half's lie.  (Rows behind the last: whatever lies there.)
  const unsigned lane16 = lane * 16;
  const bool ex = wv < 2;
  const size_t x_half = (size_t)RPx * MX_REC, w_half = (size_t)RPw * MX_REC, e_step = (size_t)(ex ? RPx : RPw) * 8;
  auto x_at = [&](int m_) { return (const char*)x + ((size_t)m_ * T::M + 64 * wv) * MX_REC; };
  auto w_at = [&](int n_) { return (const char*)w + ((size_t)n_ * T::N + 64 * wv) * MX_REC; };
  auto e_at = [&](int m_, int n_) { return (ex ? (const char*)xe + (size_t)m_ * T::M * 8 : (const char*)we + (size_t)n_ * T::N * 8) + 1024 * wn; };
  const char *px = x_at(mt), *pw = w_at(nt), *pe = e_at(mt, nt);
  auto copy_one = [&](int stage, int eslot, int i) __attribute__((always_inline)) {
    const unsigned to = lds0 + stage * T::STAGE + wv * 4096;
    if (i < 2) copy_pair(px, lane16, to, i);
    else if (i < 4) copy_pair(pw, lane16, to + T::M * MX_REC, i - 2);
    else copy_piece(pe, lane16, lds0 + AT_EXPS + eslot * T::EXPS + wv * 1024);
  };
  const int frag = l32 * MX_REC + ((hf ^ mx_swz(l32)) << 4);
  auto read_one = [&](int stage, int ks, int i, v4i (&xf)[RT], v4i (&wf)[CT]) __attribute__((always_inline)) {
    const unsigned char* s = lds + stage * T::STAGE + (frag ^ (ks << 5));
    if (i == 0) wf[0] = *(const v4i*)(s + T::M * MX_REC + CT * wn * 32 * MX_REC);
    else if (i <= RT) xf[i - 1] = *(const v4i*)(s + (RT * wm + i - 1) * 32 * MX_REC);
    else wf[i - RT] = *(const v4i*)(s + T::M * MX_REC + (CT * wn + i - RT) * 32 * MX_REC);
  };
  auto read_exp = [&](int eslot, int i, uint32_t (&xs)[RT], uint32_t (&ws)[CT]) __attribute__((always_inline)) {
    const unsigned char* s = lds + AT_EXPS + eslot * T::EXPS + 8 * l32 + 4 * hf;
    if (i < RT) xs[i] = *(const uint32_t*)(s + (RT * wm + i) * 256);
    else ws[i - RT] = *(const uint32_t*)(s + T::M * 8 + (CT * wn + i - RT) * 256);
  };

#pragma unroll
  for (int h = 0; h < STAGES; ++h) {
#pragma unroll
    for (int i = 0; i < T::COPIES + (h % 2 == 0); ++i) copy_one(h, h >> 1, i);
    px += x_half;
    pw += w_half;
    if (h % 2 == 0) pe += e_step;
  }
  // The bias of this wavefront's outputs, a tile ahead (without one what is there is copied, and not used).
  const float* const from = (const float*)(bias ? (const void*)bias : (const void*)w);
  auto copy_bias = [&](int n_) __attribute__((always_inline)) {
    copy_floats(from, 2u * (unsigned)min(n_ * T::N + 32 * CT * wn + 2 * lane, N - 2), lds0 + AT_BIAS + wv * 256);
  };
  copy_bias(nt);
  copies_barrier<0>();
  v4i x0[RT], w0[CT], x1[RT], w1[CT];
  uint32_t xx[RT], wx[CT], xn[RT], wn_[CT];
#pragma unroll
  for (int i = 0; i < OPS; ++i) read_one(0, 0, i, x0, w0);
#pragma unroll
  for (int i = 0; i < OPS; ++i) read_exp(0, i, xx, wx);
  // A tile's sums begin with the bias, by a product of its own: the bias as the first of 16 features, the tokens' a one.  (An addition of a
  // word behind the last product would be 64 instructions more for every 32 tokens, when the matrix pipe has nothing to do.)
  const uint32_t first_feature = hf == 0 ? 0xffffu : 0u, bias_mask = bias ? first_feature : 0u;
  uint32_t bias_word[CT];
  auto read_bias = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < CT; ++c) bias_word[c] = *(const uint16_t*)(lds + AT_BIAS + wv * 256 + (32 * c + l32) * 2) & bias_mask;
  };
  read_bias();
  int stage = 0, eslot = 0;
  v16f acc[RT][CT];

#define MX_PRODUCTS(KS, X, W, AFTER)                                                           \
  _Pragma("unroll") for (int i = 0; i < PRODUCTS; ++i) {                                              \
    const int c = i / RT, r = i % RT;                                                                 \
    acc[r][c] = mfma_mx<KS>(W[c], wx[c], X[r], xx[r], acc[r][c]);                                     \
    (AFTER)(i);                                                                                       \
    __builtin_amdgcn_sched_barrier(0);                                                                \
  }
// The third half on: this tile's, or the next one's.  FIRST: the first step of a tile, whose halves have all been waited for
// before the results of the tile before left (they are under way, and count like copies).
#define MX_HALF(PART, FIRST)                                                                          \
  {                                                                                                   \
    const int next = stage == STAGES - 1 ? 0 : stage + 1;                                             \
    if (PART == 1) {      /* (the half three on is the next tile's first) */                          \
      const bool turn = step == KB - 2;                                                               \
      px = turn ? next_px : px; pw = turn ? next_pw : pw; pe = turn ? next_pe : pe;                   \
    }                                                                                                 \
    _Pragma("unroll") for (int i = 0; i < 2; ++i) read_one(stage, 1, i, x1, w1);                      \
    MX_PRODUCTS(2 * PART, x0, w0, [&](int i) { if (i + 2 < OPS) read_one(stage, 1, i + 2, x1, w1); })  \
    copies_barrier<FIRST ? 63 : T::copies(PART + 2, PART + 2, 2)>();                                  \
    MX_PRODUCTS(2 * PART + 1, x1, w1, [&](int i) {                                             \
      if (i < OPS) read_one(next, 0, i, x0, w0);                                                      \
      if (PART == 1 && i < OPS) read_exp(eslot ^ 1, i, xn, wn_);                                      \
      if (i >= 3 && i % 2 == 1 && (i - 3) / 2 < T::COPIES + PART) copy_one(stage, eslot, (i - 3) / 2);  \
    })                                                                                                \
    px += x_half;                                                                                     \
    pw += w_half;                                                                                     \
    if (PART == 1) pe += e_step;                                                                      \
    if constexpr (PART == 1) {                                                                        \
      _Pragma("unroll") for (int r = 0; r < RT; ++r) xx[r] = xn[r];                                   \
      _Pragma("unroll") for (int c = 0; c < CT; ++c) wx[c] = wn_[c];                                  \
      eslot ^= 1;                                                                                     \
    }                                                                                                 \
    stage = next;                                                                                     \
  }
  while (true) {
    const int next_slot = slot + walkers;
    const bool more = next_slot < tiles.n;
    tiles.at(more ? next_slot : slot, next_mt, next_nt);   // (behind the last tile its first halves once more, for nobody)
    const char *const next_px = x_at(next_mt), *const next_pw = w_at(next_nt), *const next_pe = e_at(next_mt, next_nt);
    const int n0 = nt * T::N + 32 * CT * wn;
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int r = 0; r < RT; ++r)
        acc[r][c] = mfma_bf16(uint4{bias_word[c], 0u, 0u, 0u}, uint4{first_feature & 0x3f80u, 0u, 0u, 0u}, v16f{});
    __builtin_amdgcn_sched_barrier(0);
    int step = 0;
    MX_HALF(0, true)
    copy_bias(next_nt);                  // (its words have been read: the meeting in the half before waited for them)
    MX_HALF(1, true)
    for (step = 1; step < KB; ++step) {
      MX_HALF(0, false)
      MX_HALF(1, false)
    }
    // Results: bf16, through LDS of their own so that rows leave as whole lines, past the caches.  The stores go by a buffer
    // that ends with the last token and drops what lies behind its end: no branch may stand here, or the sums would be moved out of
    // their registers all at once.
    int ln = lane;
    asm volatile("" : "+v"(ln));         // (nothing of this part is worth a register in the loop)
    const int q32 = ln & 31, qh = ln >> 5, part = ln & 15, row0 = mt * T::M + 32 * RT * wm;
    unsigned char* my = lds + AT_OUT + wv * (32 * T::EPI);
    const unsigned left = (unsigned)max(0, min(M - row0, 32 * RT)) * (2u * (unsigned)N);
    const uint64_t first = (uint64_t)(uintptr_t)(y + (size_t)row0 * N);      // (uniform, which the compiler does not see)
    const uint64_t base = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(first >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)first);
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, __builtin_amdgcn_readfirstlane((int)left), 0x00020000);
    const unsigned at = n0 + 8 * part < N ? (unsigned)(ln >> 4) * (2u * (unsigned)N) + 2u * (n0 + 8 * part) : 0x80000000u;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
      for (int c = 0; c < CT; ++c) asm volatile("" : "+a"(acc[r][c]));   // (not earlier than here)
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const v16f& f = acc[r][c];
          *(uint2*)(my + q32 * T::EPI + (32 * c + 8 * g + 4 * qh) * 2) =
              make_uint2(pack_bf16x2(f[4 * g], f[4 * g + 1]), pack_bf16x2(f[4 * g + 2], f[4 * g + 3]));
        }
      // (the next tile's first halves: waited for before the first result leaves, behind which they could not be told from it)
      if (r == 0) {
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        read_bias();
      }
      __builtin_amdgcn_wave_barrier();   // (a wavefront's LDS operations execute in order: only the compiler has to keep it)
      v4i out[8];
#pragma unroll
      for (int it = 0; it < 8; ++it) out[it] = *(const v4i*)(my + (it * 4 + (ln >> 4)) * T::EPI + part * 16);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int it = 0; it < 8; ++it)     // (2: past the caches)
        __builtin_amdgcn_raw_buffer_store_b128(out[it], buffer, at + (unsigned)(32 * r + 4 * it) * (2u * (unsigned)N), 0, 2);
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!more) break;
    slot = next_slot;
    mt = next_mt;
    nt = next_nt;
  }
#undef MX_HALF
#undef MX_PRODUCTS
}

template <int WM, int WN, int RT, int CT, int STAGES, int PER_CU>
static void launch_tiles(const uint8_t* x, const uint8_t* xe, const uint8_t* w, const uint8_t* we, const void* bias, void* y, int M,
                         int N, int K, hipStream_t stream) {
  using T = MxTile<WM, WN, RT, CT, STAGES>;
  const int MT = (M + T::M - 1) / T::M, NT = (N + T::N - 1) / T::N;
  const unsigned grid = (unsigned)(8 * (MT >= MX_DEAL_MT ? (MT + 7) / 8 * NT : (MT * NT + 7) / 8));
  mxfp4_gemm_kernel<WM, WN, RT, CT, STAGES, PER_CU><<<grid, 256, 0, stream>>>(
      x, xe, w, we, (const bf16_t*)bias, (bf16_t*)y, M, N, mx_steps(K), MT, NT);
}

// ---------------------------------------------------------------------------
// Sixteen rows a wavefront, two where that would leave compute units without work.
#define MX_ROWS(KERNEL, ...)                                                                                          \
  do {                                                                                                                \
    const int KB = mx_steps(K), pairs = (long long)((R + 15) / 16) * KB >= 4096 ? 8 : 1;                              \
    const int units = (R + 2 * pairs - 1) / (2 * pairs) * KB;                                                         \
    const unsigned grid = (unsigned)((units + 3) / 4);                                                                \
    if (pairs == 1) KERNEL<1, false><<<grid, 256, 0, stream>>>(__VA_ARGS__);                                          \
    else if ((long long)R * K * 2 > (256ll << 20)) KERNEL<8, true><<<grid, 256, 0, stream>>>(__VA_ARGS__);            \
    else KERNEL<8, false><<<grid, 256, 0, stream>>>(__VA_ARGS__);                                                     \
  } while (0)
void launch_mxfp4_quantize(const void* x, int R, int K, uint8_t* codes, uint8_t* exps, hipStream_t stream) {
  MX_ROWS(mxfp4_quantize_kernel, (const bf16_t*)x, R, K, mx_rows(R), KB, units, codes, exps);
}
void launch_mxfp4_dequantize(const uint8_t* codes, const uint8_t* exps, int R, int K, void* x, hipStream_t stream) {
  MX_ROWS(mxfp4_dequantize_kernel, codes, exps, R, K, mx_rows(R), KB, units, (bf16_t*)x);
}
#undef MX_ROWS
void launch_mxfp4_pack(const uint8_t* from, const uint8_t* from_exps, int R, int K, uint8_t* codes, uint8_t* exps, hipStream_t stream) {
  mxfp4_pack_kernel<<<2048, 256, 0, stream>>>(from, from_exps, R, K, mx_rows(R), mx_steps(K), codes, exps);
}
void launch_mxfp4_unpack(const uint8_t* codes, const uint8_t* exps, int R, int K, uint8_t* to, uint8_t* to_exps, hipStream_t stream) {
  mxfp4_unpack_kernel<<<2048, 256, 0, stream>>>(codes, exps, R, K, mx_rows(R), to, to_exps);
}
template <int RT, int CT, int KSPLIT, bool QUANT = false>
static void launch_split(const uint8_t* x, const uint8_t* xe, const uint8_t* w, const uint8_t* we, const void* bias, void* y, int M,
                         int N, int K, hipStream_t stream) {
  const int MT = (M + 32 * RT - 1) / (32 * RT), NT = (N + 32 * CT - 1) / (32 * CT);
  mxfp4_gemm_split_kernel<RT, CT, KSPLIT, QUANT><<<8u * (((unsigned)MT * NT + 7) / 8), 64 * KSPLIT, 0, stream>>>(
      x, xe, w, we, (const bf16_t*)bias, (bf16_t*)y, M, N, K, mx_steps(K), MT, NT);
}

// Which kernel.  Products alone in us, in a captured graph (walk: 256 x 256 walked; wide: 256 x 128, two to a compute unit; square: 128 x
// 128 with 3 or 4 stages, three or two to a compute unit; split: RT, CT, wavefronts):
//   walk from 1024 of its tiles and four steps on: 16384 x 5120 -> 5120 (1280) walk 191, wide 200, 20000 x 1536 -> 8960 (2765) 156 / 158; 12000 x
//   1536 -> 4608 (846) 59.6 / 48.1, 8192 x 5120 -> 5120 (640) 119 / 113, 65536 x 640 -> 1280 (1280) 47.9 / 46.5;
//   wide from 512 of its tiles on: 4096 x 5120 -> 5120 (640) wide 54.9, square 57.1, walk 65; 2048 x 5120 -> 5120 (320) 33.2 / 31.8 / 32.4;
//   fewer of the larger tiles where the contraction is long and the busiest compute unit has no more to do with them: walk 5000 x 13824 -> 5120
//   (400) 168, wide (800) 181, 2048 x 5120 -> 13824 (432) 71.1 / 74.5, 4096 x 5120 -> 15360 (960) 147 / 152, but 2000 x 2560 -> 15360 (480) 44.6 / 43.6
//   and 8192 x 8960 -> 5120 (640, 3 rounds to 5) 167 / 164; wide 1024 x 5120 -> 13824 (432) 37.0, square (864) 41.6, 1024 x 8960 -> 5120 (160) 28.1 /
//   31.1, 512 x 2560 -> 13824 (216) 12.9 / 13.1, but 1024 x 2048 -> 8192 (256) 12.1 / 10.9, 1800 x 5120 -> 5120 (320 to 600, 2 rounds to 3) 32.6 / 30.6;
//   square from 64 tiles on: 1024 x 1536 -> 1536 (96) square 6.0, split 6.9; 256 x 5120 -> 5120 (80) 11.9 / 14.1; 300 x 2560 -> 2560 (60) 7.4 /
//   6.2; 128 x 5120 -> 5120 (40) 11.4 / 8.7; with four stages up to 256 tiles: 512 x 5120 -> 5120 (160) 12.7 against 13.5, 700 x 8960 -> 1536
//   (72) 18.4 / 20.6, but 1024 x 5120 -> 5120 (320) 22.1 / 20.9;
//   split: 64 x 5120 -> 5120 2, 2, 4: 8.7, 1, 2, 4: 7.3; 1 x 5120 -> 5120 1, 1, 4: 5.3, 1, 1, 8: 5.1, 16 x 1536 -> 8960 4.0 / 4.1.
void launch_mxfp4_gemm(const uint8_t* x, const uint8_t* xe, const uint8_t* w, const uint8_t* we, const void* bias, void* y, int M,
                       int N, int K, hipStream_t stream) {
  auto tiles = [&](int m, int n) { return (long long)((M + m - 1) / m) * ((N + n - 1) / n); };
  // what the busiest compute unit has to do, in square tiles
  auto load = [&](int m, int n) { return m * n / 16384 * ((tiles(m, n) + 255) / 256); };
  const bool deep = K > 8 * MX_STEP;
  if ((K > 3 * MX_STEP && tiles(256, 256) >= 1024) ||
      (deep && load(256, 256) <= load(256, 128) && 6 * load(256, 256) <= 7 * load(128, 128))) {
    // (256 workgroups: one to a compute unit, a multiple of the 8 XCDs)
    mxfp4_gemm_walk_kernel<<<256, 256, 0, stream>>>(x, xe, w, we, (const bf16_t*)bias, (bf16_t*)y, M, N, mx_steps(K), (M + 255) / 256, (N + 255) / 256);
    return;
  }
#define MX_ARGS x, xe, w, we, bias, y, M, N, K, stream
  if (M <= 64) {
    if (M > 32) return launch_split<1, 2, 4>(MX_ARGS);
    if (K > 16 * MX_STEP) return launch_split<1, 1, 8>(MX_ARGS);
    return launch_split<1, 1, 4>(MX_ARGS);
  }
  if (tiles(256, 128) >= 512 || (deep && load(256, 128) <= load(128, 128))) return launch_tiles<4, 1, 2, 4, 3, 2>(MX_ARGS);
  if (tiles(128, 128) > 256) return launch_tiles<2, 2, 2, 2, 3, 3>(MX_ARGS);
  if (tiles(128, 128) >= 64) return launch_tiles<2, 2, 2, 2, 4, 2>(MX_ARGS);
  launch_split<2, 2, 4>(MX_ARGS);
#undef MX_ARGS
}

// The layer of bf16 tokens where they are so few that every workgroup quantises them by itself; false: not such a call.  In us, in a
// captured graph, against two launches: 1 x 5120 -> 5120 5.0 / 7.7, 4 x 5120 6.1 / 7.9, 1 x 1536 -> 8960 3.7 / 7.3, 16 x 1536 7.3 / 8.3, 32 x 1000
// -> 1000 6.1 / 6.1; beyond, 24 x 1536 -> 8960 9.4 / 8.4, 8 x 5120 -> 5120 7.9 / 8.4.
bool launch_mxfp4_linear_few(const void* x, const uint8_t* w, const uint8_t* we, const void* bias, void* y, int M, int N, int K,
                             hipStream_t stream) {
  if (M > 32 || M * mx_steps(K) * MX_STEP > MX_FEW) return false;
  if (K > 16 * MX_STEP) launch_split<1, 1, 8, true>((const uint8_t*)x, nullptr, w, we, bias, y, M, N, K, stream);
  else launch_split<1, 1, 4, true>((const uint8_t*)x, nullptr, w, we, bias, y, M, N, K, stream);
  return true;
}

}  // namespace sla
