// Microscaled 4-bit floating point (include/mxfp4.h): quantisation, its inverse, plain rows from and into the operand order
// (mxfp4.h), and the product of two quantised matrices.
#include "mxfp4.h"
#include "rows.h"
#include "tiles.h"

namespace sla {

// ---------------------------------------------------------------------------
// A wavefront takes 512 features of ROWS rows, eight features a lane: four lanes are a block.
template <int ROWS>
__global__ void __launch_bounds__(256) mxfp4_quantize_kernel(const bf16_t* __restrict__ x, int R, int K, int RP, int KB,
                                                             uint8_t* __restrict__ codes, uint8_t* __restrict__ exps) {
  const int halves = (KB + 1) / 2, unit = (int)blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int group = unit / halves, k8 = (unit - group * halves) * 64 + lane, r0 = group * ROWS;
  if (r0 >= R || k8 >= KB * (MX_STEP / 8)) return;
  uint4 v[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    v[i] = uint4{0u, 0u, 0u, 0u};
    if (r0 + i < R && k8 < K / 8) v[i] = *(const uint4*)(x + (long long)(r0 + i) * K + 8ll * k8);
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
    if (r0 + i < R) mx_store8(v[i], r0 + i, k8, RP, codes, exps);
}

// Eight features a thread.
__global__ void __launch_bounds__(256) mxfp4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ exps,
                                                               int R, int K, int RP, bf16_t* __restrict__ x) {
  const int halves = (K / 8 + 63) / 64, unit = (int)blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = unit / halves, k8 = (unit - row * halves) * 64 + lane;
  if (row >= R || k8 >= K / 8) return;
  const int kb = k8 >> 5, c = (k8 >> 2) & 7;
  const uint32_t four = *(const uint32_t*)(codes + mx_chunk_at(RP, row, kb, c) + 4 * (k8 & 3));
  const uint32_t e = exps[mx_exp_at(RP, row, kb, c)];
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = (four >> (4 * i)) & 7u, sign = (four >> (4 * i + 3)) << 31;
    // twice the magnitude: 0, 1, 2, 3, 4, 6, 8, 12
    const float twice = m < 4 ? (float)m : (float)((4 + 2 * (m & 1)) << ((m >> 1) - 2));
    v[i] = e == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(__float_as_uint(ldexpf(twice, (int)e - 128)) | sign);
  }
  *(uint4*)(x + (long long)row * K + 8ll * k8) = pack8(v);
}

// One block of 32 features a thread.
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

// Workgroup tile (32 RT) tokens x (32 CT) outputs; its KSPLIT wavefronts split the contraction and meet in LDS in a fixed order.
// Operands go from memory straight to registers.
template <int RT, int CT, int KSPLIT>
__global__ void __launch_bounds__(64 * KSPLIT) mxfp4_gemm_split_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xe,
                                                                       const uint8_t* __restrict__ w, const uint8_t* __restrict__ we,
                                                                       const bf16_t* __restrict__ bias, bf16_t* __restrict__ y, int M,
                                                                       int N, int KB, int MT, int NT) {
  constexpr int PITCH = 36;  // floats per staged row of 32 outputs (16-byte rows, skewed banks)
  __shared__ __attribute__((aligned(16))) float part[KSPLIT][32 * RT][PITCH];
  const int mt = blockIdx.x % MT, nt = blockIdx.x / MT;
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
  for (int kb = kb0; kb < kb1; ++kb) {
    v4i a[CT][4], b[RT][4];
    uint32_t ae[CT], be[RT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const int row = row_of(nt * CT + c, RPw);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) a[c][ks] = *(const v4i*)(w + mx_chunk_at(RPw, row, kb, 2 * ks + hf));
      ae[c] = *(const uint32_t*)(we + mx_exp_at(RPw, row, kb, hf));
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int row = row_of(mt * RT + r, RPx);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) b[r][ks] = *(const v4i*)(x + mx_chunk_at(RPx, row, kb, 2 * ks + hf));
      be[r] = *(const uint32_t*)(xe + mx_exp_at(RPx, row, kb, hf));
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        acc[r][c] = mfma_mx<0>(a[c][0], ae[c], b[r][0], be[r], acc[r][c]);
        acc[r][c] = mfma_mx<1>(a[c][1], ae[c], b[r][1], be[r], acc[r][c]);
        acc[r][c] = mfma_mx<2>(a[c][2], ae[c], b[r][2], be[r], acc[r][c]);
        acc[r][c] = mfma_mx<3>(a[c][3], ae[c], b[r][3], be[r], acc[r][c]);
      }
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
// Large calls: workgroup tile 256 tokens x 128 outputs, four wavefronts of 64 x 128, two workgroups per compute unit.  Half a step
// (128 features: 24 KiB of records) is a stage; three stages are in LDS, copied without registers in between; a step's exponents
// (3 KiB) ride with its first half, in two places of their own.
// A half's first 64 features are read while the second ones of the half before are multiplied; in the middle of a half, when all
// of its operands are in registers, the workgroup meets: behind that its stage is free for the half three on, and the next half's
// has arrived.
// ---------------------------------------------------------------------------
constexpr int MX_WG_M = 256, MX_WG_N = 128;
constexpr int MX_STAGE = (MX_WG_M + MX_WG_N) * MX_REC, MX_EXPS = (MX_WG_M + MX_WG_N) * 8;
constexpr int MX_EPI_STRIDE = MX_WG_N * 2 + 16;   // bytes per staged output row
constexpr int MX_DEAL_MT = 64;                    // token tiles from which whole ones are dealt to the XCDs

__global__ void __launch_bounds__(256, 2) mxfp4_gemm_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xe,
                                                            const uint8_t* __restrict__ w, const uint8_t* __restrict__ we,
                                                            const bf16_t* __restrict__ bias, bf16_t* __restrict__ y, int M, int N,
                                                            int KB, int MT, int NT) {
  __shared__ __attribute__((aligned(1024))) unsigned char lds[3 * MX_STAGE + 2 * MX_EXPS];
  static_assert(4 * 32 * MX_EPI_STRIDE <= 3 * MX_STAGE, "output staging fits the stages");
  // Workgroups are dealt round-robin over the 8 XCDs.  An XCD walks its tiles in patches of 8 x 8, what its 32 compute units hold
  // at a time, so that each record of a step is fetched into its L2 once for eight users; of many token tiles it takes every
  // eighth, of few an eighth of all tiles.
  const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const bool deal = MT >= MX_DEAL_MT;
  const int share = (MT * NT + 7) >> 3, first = deal ? 0 : xcd * share, rows = deal ? (MT - xcd + 7) >> 3 : MT;
  if (slot >= (deal ? rows * NT : min(share, MT * NT - first))) return;
  const int idx = first + slot, band = idx / (8 * NT), in_band = idx - band * 8 * NT, band_rows = min(8, rows - 8 * band);
  const int grp = in_band / (8 * band_rows), in_grp = in_band - grp * 8 * band_rows;
  const int cols = min(8, NT - 8 * grp), trow = 8 * band + in_grp / cols;
  const int mt = __builtin_amdgcn_readfirstlane(deal ? 8 * trow + xcd : trow);
  const int nt = __builtin_amdgcn_readfirstlane(8 * grp + in_grp % cols);

  const int t = threadIdx.x, lane = t & 63, wv = __builtin_amdgcn_readfirstlane(t >> 6), l32 = lane & 31, hf = lane >> 5;
  const int RPx = mx_rows(M), RPw = mx_rows(N), H = 2 * KB;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)lds;

  // This wavefront's copies of a half: four pieces (16 records each) of its tokens, two of the weight; of a step's exponents one
  // (128 rows; the fourth wavefront repeats the third's).  Rows behind the last: the last ones once more.
  unsigned xo[4], wo[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) xo[i] = (unsigned)min(mt * MX_WG_M + 64 * wv + 16 * i, RPx - 16) * MX_REC + lane * 16;
#pragma unroll
  for (int i = 0; i < 2; ++i) wo[i] = (unsigned)min(nt * MX_WG_N + 32 * wv + 16 * i, RPw - 16) * MX_REC + lane * 16;
  const bool ex = wv < 2;
  const unsigned eo = (unsigned)(ex ? min(mt * MX_WG_M + 128 * wv + 2 * lane, RPx - 2) : min(nt * MX_WG_N + 2 * lane, RPw - 2)) * 8;
  const char* const e_base = (const char*)(ex ? xe : we);
  const size_t e_step = (size_t)(ex ? RPx : RPw) * 8;
  auto copy_half = [&](int h, int stage, bool with_exps) __attribute__((always_inline)) {
    const char *xs = (const char*)x + (size_t)h * RPx * MX_REC, *ws = (const char*)w + (size_t)h * RPw * MX_REC;
    const unsigned to = lds0 + stage * MX_STAGE;
#pragma unroll
    for (int i = 0; i < 4; ++i) copy_piece(xs, xo[i], to + (4 * wv + i) * 1024);
#pragma unroll
    for (int i = 0; i < 2; ++i) copy_piece(ws, wo[i], to + MX_WG_M * MX_REC + (2 * wv + i) * 1024);
    if (with_exps) copy_piece(e_base + (h >> 1) * e_step, eo, lds0 + 3 * MX_STAGE + ((h >> 1) & 1) * MX_EXPS + min(wv, 2) * 1024);
  };
  // operands: token tiles 2 wv + r, output tiles c
  const int frag = l32 * MX_REC + ((hf ^ mx_swz(l32)) << 4);
  auto read_half = [&](int stage, int ks, v4i (&xf)[2], v4i (&wf)[4]) __attribute__((always_inline)) {
    const unsigned char* s = lds + stage * MX_STAGE + (frag ^ (ks << 5));
#pragma unroll
    for (int r = 0; r < 2; ++r) xf[r] = *(const v4i*)(s + (2 * wv + r) * 32 * MX_REC);
#pragma unroll
    for (int c = 0; c < 4; ++c) wf[c] = *(const v4i*)(s + MX_WG_M * MX_REC + c * 32 * MX_REC);
  };
  uint32_t xx[2], wx[4];
  auto read_exps = [&](int step) __attribute__((always_inline)) {
    const unsigned char* s = lds + 3 * MX_STAGE + (step & 1) * MX_EXPS + 8 * l32 + 4 * hf;
#pragma unroll
    for (int r = 0; r < 2; ++r) xx[r] = *(const uint32_t*)(s + (2 * wv + r) * 256);
#pragma unroll
    for (int c = 0; c < 4; ++c) wx[c] = *(const uint32_t*)(s + MX_WG_M * 8 + c * 256);
  };
  v16f acc[2][4];
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[r][c] = v16f{};

  copy_half(0, 0, true);
  copy_half(1, 1, false);
  if (H > 2) {
    copy_half(2, 2, true);
    copies_barrier<13>();
  } else {
    copies_barrier<6>();
  }
  v4i x0[2], w0[4], x1[2], w1[4];
  read_half(0, 0, x0, w0);
  read_exps(0);
  int stage = 0;
#define MX_PRODUCTS(KS, X, W)                                                                    \
  _Pragma("unroll") for (int c = 0; c < 4; ++c)                                                  \
  _Pragma("unroll") for (int r = 0; r < 2; ++r) acc[r][c] = mfma_mx<KS>(W[c], wx[c], X[r], xx[r], acc[r][c]); \
  __builtin_amdgcn_sched_barrier(0);
// (LEFT: steps behind this one, 2 for two or more.  A step is free of branches: the compiler would move the products past them.)
#define MX_HALF(PART, LEFT)                                                                      \
  {                                                                                              \
    const int h = 2 * step + PART, next = stage == 2 ? 0 : stage + 1;                            \
    read_half(stage, 1, x1, w1);                                                                 \
    __builtin_amdgcn_sched_barrier(0);                                                           \
    MX_PRODUCTS(2 * PART, x0, w0)                                                                \
    copies_barrier<LEFT == 0 ? 0 : PART == 0 ? 7 : 6>();                                         \
    if constexpr (LEFT + PART >= 2 ? LEFT == 2 : LEFT == 1) copy_half(h + 3, stage, PART == 1);  \
    if constexpr (LEFT > 0 || PART == 0) read_half(next, 0, x0, w0);                             \
    __builtin_amdgcn_sched_barrier(0);                                                           \
    MX_PRODUCTS(2 * PART + 1, x1, w1)                                                            \
    if constexpr (LEFT > 0 && PART == 1) read_exps(step + 1);                                    \
    stage = next;                                                                                \
  }
  int step = 0;
  for (; step + 2 < KB; ++step) {
    MX_HALF(0, 2)
    MX_HALF(1, 2)
  }
  if (KB > 1) {
    MX_HALF(0, 1)
    MX_HALF(1, 1)
    ++step;
  }
  MX_HALF(0, 0)
  MX_HALF(1, 0)
#undef MX_HALF
#undef MX_PRODUCTS

  // Epilogue: bias in, bf16, through LDS so that rows leave as 256 contiguous bytes, past the caches.  (Behind the last meeting
  // nobody reads the stages for a result.)
  unsigned char* my = lds + wv * (32 * MX_EPI_STRIDE);
  const int n0 = nt * MX_WG_N;
  uint2 bw[4][4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g) bw[c][g] = make_uint2(0u, 0u);
  if (bias) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g) bw[c][g] = *(const uint2*)(bias + min(n0 + 32 * c + 8 * g + 4 * hf, N - 4));
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint2 b4 = bw[c][g];
        const v16f& f = acc[r][c];
        *(uint2*)(my + l32 * MX_EPI_STRIDE + (32 * c + 8 * g + 4 * hf) * 2) =
            make_uint2(pack_bf16x2(f[4 * g] + bf16_lo(b4.x), f[4 * g + 1] + bf16_hi(b4.x)),
                       pack_bf16x2(f[4 * g + 2] + bf16_lo(b4.y), f[4 * g + 3] + bf16_hi(b4.y)));
      }
    __builtin_amdgcn_wave_barrier();     // (a wavefront's LDS operations execute in order: only the compiler has to keep it)
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const int row = it * 4 + (lane >> 4), part = lane & 15;
      const int m = mt * MX_WG_M + 64 * wv + 32 * r + row;
      const v4i v = *(const v4i*)(my + row * MX_EPI_STRIDE + part * 16);
      if (m < M && n0 + 8 * part < N) __builtin_nontemporal_store(v, (v4i*)(y + (size_t)m * N + n0 + part * 8));
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// ---------------------------------------------------------------------------
void launch_mxfp4_quantize(const void* x, int R, int K, uint8_t* codes, uint8_t* exps, hipStream_t stream) {
  const int KB = mx_steps(K);
  const long long units = (long long)((R + 7) / 8) * ((KB + 1) / 2);
  mxfp4_quantize_kernel<8><<<(unsigned)((units + 3) / 4), 256, 0, stream>>>((const bf16_t*)x, R, K, mx_rows(R), KB, codes, exps);
}
void launch_mxfp4_dequantize(const uint8_t* codes, const uint8_t* exps, int R, int K, void* x, hipStream_t stream) {
  const long long units = (long long)R * ((K / 8 + 63) / 64);
  mxfp4_dequantize_kernel<<<(unsigned)((units + 3) / 4), 256, 0, stream>>>(codes, exps, R, K, mx_rows(R), (bf16_t*)x);
}
void launch_mxfp4_pack(const uint8_t* from, const uint8_t* from_exps, int R, int K, uint8_t* codes, uint8_t* exps, hipStream_t stream) {
  mxfp4_pack_kernel<<<2048, 256, 0, stream>>>(from, from_exps, R, K, mx_rows(R), mx_steps(K), codes, exps);
}
void launch_mxfp4_unpack(const uint8_t* codes, const uint8_t* exps, int R, int K, uint8_t* to, uint8_t* to_exps, hipStream_t stream) {
  mxfp4_unpack_kernel<<<2048, 256, 0, stream>>>(codes, exps, R, K, mx_rows(R), to, to_exps);
}
void launch_mxfp4_gemm(const uint8_t* x, const uint8_t* xe, const uint8_t* w, const uint8_t* we, const void* bias, void* y, int M,
                       int N, int K, hipStream_t stream) {
  {
    const int MT = (M + MX_WG_M - 1) / MX_WG_M, NT = (N + MX_WG_N - 1) / MX_WG_N;
    if (MT * NT >= 256) {
      const unsigned grid = (unsigned)(8 * (MT >= MX_DEAL_MT ? (MT + 7) / 8 * NT : (MT * NT + 7) / 8));
      mxfp4_gemm_kernel<<<grid, 256, 0, stream>>>(x, xe, w, we, (const bf16_t*)bias, (bf16_t*)y, M, N, mx_steps(K), MT, NT);
      return;
    }
  }
  const int MT = (M + 63) / 64, NT = (N + 63) / 64;
  mxfp4_gemm_split_kernel<2, 2, 4><<<(unsigned)MT * NT, 256, 0, stream>>>(x, xe, w, we, (const bf16_t*)bias, (bf16_t*)y, M, N, mx_steps(K), MT, NT);
}

}  // namespace sla
