// The operand order of a matrix in microscaled 4-bit floating point (include/mxfp4.h), and a block's quantisation.
//
// A matrix of R rows and K features, RP = R rounded up to 32 and KP = K rounded up to 256, is stored as records of 64 bytes,
// [KP / 128][RP]: 128 features of a row, two to a byte (the first in the low half), in four chunks of 16 bytes, one per
// block of 32; chunk c of row r stands at position c ^ (r / 4 & 3).  Copied to LDS as they are, 32 rows are then read by a
// wavefront's 64 lanes without bank conflicts (16 lanes that read chunk c of 16 rows meet all 64 banks once).
// The exponents follow, [KP / 256][RP] of 8 bytes: that of block 2 ks + hf at byte 4 hf + ks, so that the word of lane half hf
// holds what v_mfma_scale_f32_32x32x64_f8f6f4 takes for its four steps ks.  Blocks behind the last feature have codes 0 and
// the smallest exponent; rows behind the last hold anything (they meet only results that are not stored).
#pragma once
#include "common.h"

namespace sla {

constexpr int MX_BLOCK = 32, MX_STEP = 256, MX_REC = 64;
__host__ __device__ inline int mx_rows(int R) { return (R + 31) / 32 * 32; }
__host__ __device__ inline int mx_steps(int K) { return (K + MX_STEP - 1) / MX_STEP; }
inline size_t mx_codes_bytes(int R, int K) { return align256((size_t)mx_rows(R) * mx_steps(K) * (MX_STEP / 2)); }
// (the product copies whole tiles of up to 256 rows: behind the last row it reads what follows, at most the records of so many
// rows behind the end)
constexpr int MX_TILE_ROWS = 256;
inline size_t mx_object_bytes(int R, int K) {
  return mx_codes_bytes(R, K) + align256((size_t)mx_rows(R) * mx_steps(K) * 8) + MX_TILE_ROWS * MX_REC;
}

// byte of the chunk of block c (0..7) of a row's 256 features kb, and of its exponent
__device__ __forceinline__ int mx_swz(int row) { return (row >> 2) & 3; }
__device__ __forceinline__ size_t mx_chunk_at(int RP, int row, int kb, int c) {
  return ((size_t)(2 * kb + (c >> 2)) * RP + row) * MX_REC + (((c & 3) ^ mx_swz(row)) << 4);
}
__device__ __forceinline__ size_t mx_exp_at(int RP, int row, int kb, int c) { return ((size_t)kb * RP + row) * 8 + 4 * (c & 1) + (c >> 1); }

// The exponent's byte of a block whose largest magnitude is amax: floor(log2 amax) - 2, so that the quotients stay below 8, at
// least -126 (the quotient's scale is then a normal number); 255 where amax is infinite or NaN.
__device__ __forceinline__ uint32_t mx_exponent(float amax) {
  const int e = (int)((__float_as_uint(amax) >> 23) & 255u);
  return e == 255 ? 255u : (uint32_t)max(e - 2, 1);
}
// Codes of eight bf16 features (the words of 16 bytes), the first in the lowest bits; no code of a block that is no number.
__device__ __forceinline__ uint32_t mx_codes8(const uint4& v, uint32_t exponent) {
  const float s = __uint_as_float(exponent << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf, v.x), s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf, v.y), s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf, v.z), s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(v2bf, v.w), s, 3);
  return exponent == 255u ? 0u : c;
}
// The largest magnitude of eight bf16 features; an infinity or a NaN among them comes out as one of the two.
__device__ __forceinline__ float mx_amax8(const uint4& v) {
  // (magnitudes as integers: ordered like the numbers, infinities and NaNs last)
  const uint32_t w[4] = {v.x & 0x7fff7fffu, v.y & 0x7fff7fffu, v.z & 0x7fff7fffu, v.w & 0x7fff7fffu};
  uint32_t lo = 0, hi = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo = max(lo, w[i] << 16);
    hi = max(hi, w[i] & 0xffff0000u);
  }
  return __uint_as_float(max(lo, hi));
}
// The same over a quad of lanes, whose 32 features are a block.
__device__ __forceinline__ uint32_t quad_umax(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));
}
// Eight features of a row (number k8 of them, its block the quad's) to their place.
__device__ __forceinline__ void mx_store8(const uint4& v, int row, int k8, int RP, uint8_t* codes, uint8_t* exps) {
  const uint32_t e = mx_exponent(__uint_as_float(quad_umax(__float_as_uint(mx_amax8(v)))));
  const int kb = k8 >> 5, c = (k8 >> 2) & 7, part = k8 & 3;
  *(uint32_t*)(codes + mx_chunk_at(RP, row, kb, c) + 4 * part) = mx_codes8(v, e);
  if (part == 0) exps[mx_exp_at(RP, row, kb, c)] = (uint8_t)e;
}

}  // namespace sla
