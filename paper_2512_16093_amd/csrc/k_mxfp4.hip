// Microscaled 4-bit floating point (include/mxfp4.h): quantisation, its inverse, plain rows from and into the operand order
// (mxfp4.h), and the product of two quantised matrices.
#include "mxfp4.h"
#include "rows.h"

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
      const size_t rec = (size_t)kb * RPw + row_of(nt * CT + c, RPw);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) a[c][ks] = *(const v4i*)(w + rec * MX_REC + (((2 * ks + hf) ^ (l32 & 7)) << 4));
      ae[c] = *(const uint32_t*)(we + rec * 8 + 4 * hf);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const size_t rec = (size_t)kb * RPx + row_of(mt * RT + r, RPx);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) b[r][ks] = *(const v4i*)(x + rec * MX_REC + (((2 * ks + hf) ^ (l32 & 7)) << 4));
      be[r] = *(const uint32_t*)(xe + rec * 8 + 4 * hf);
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
  const int MT = (M + 63) / 64, NT = (N + 63) / 64;
  mxfp4_gemm_split_kernel<2, 2, 4><<<(unsigned)MT * NT, 256, 0, stream>>>(x, xe, w, we, (const bf16_t*)bias, (bf16_t*)y, M, N, mx_steps(K), MT, NT);
}

}  // namespace sla
