// Token rows as operands of the matrix products: a wavefront's own rows straight from memory, tiles of 32 rows x 128 channels
// copied to LDS without registers in between and read from there.
#pragma once
#include "common.h"

namespace sla {

// The same operand as n_op straight from memory (a workgroup's own rows, read once).
// (x: the (b,h) slice's first token; sn: elements from one token to the next)
__device__ __forceinline__ void own_rows(const bf16_t* x, long long sn, long long row, int N, int hf, uint4 (&f)[8]) {
#pragma unroll
  for (int ks = 0; ks < 8; ++ks) f[ks] = row < N ? *(const uint4*)(x + row * sn + 16 * ks + 8 * hf) : uint4{0u, 0u, 0u, 0u};
}
// First token of slice bh = b H + h of a tensor laid out by L.
__device__ __forceinline__ const bf16_t* slice_of(const bf16_t* x, const Layout& L, int bh, int H) {
  const int b = bh / H;
  return x + b * L.sb + (bh - b * H) * L.sh;
}
__device__ __forceinline__ bf16_t* slice_of(bf16_t* x, const Layout& L, int bh, int H) {
  const int b = bh / H;
  return x + b * L.sb + (bh - b * H) * L.sh;
}

// ---- asynchronous copies of 32-row tiles (32 x 256 bytes) global -> LDS, without registers in between
//
// A tile is eight pieces of 1 KiB (four rows); a wavefront's copy instruction writes one piece, lane l its bytes
// [16 l, 16 l + 16).  The copy cannot pad rows, so a row's sixteen 16-byte chunks are stored permuted, chunk c of row r
// at position c ^ swz(r): the 16 lanes of a group that read the same chunk of 16 consecutive rows hit all banks once
// (n_op_swz), and so do the 32 lanes that read a 4-row x 64-byte patch (t_op_swz).  The compiler does not know these
// copies are in flight (it would wait for all of them before every LDS read): the callers wait by count.
constexpr int SWZ_TILE_B = 32 * 256;
__device__ __forceinline__ int swz(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }
__device__ __forceinline__ void copy_piece(const char* base, unsigned off, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %0" : : "s"(base), "v"(off), "s"(lds_addr) : "memory", "m0");
}
__device__ __forceinline__ void copy_piece(const char* addr, unsigned lds_addr) {  // (an address per lane)
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(addr), "s"(lds_addr) : "memory", "m0");
}
// Two consecutive pieces of a tile (FIRST and the next one), of no lane (mask 0) or all of them (-1; no wavefront here ever
// has a lane switched off).  The instruction's immediate offset moves both addresses, so lds_tile is that of the
// wavefront's first piece and base, off as TileCopy::base3 and off3 give them.
template <int FIRST>
__device__ __forceinline__ void copy_pieces_if(long long mask, const char* base, unsigned off0, unsigned off1, unsigned lds_tile) {
  asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 exec, %4\n\t"
               "global_load_lds_dwordx4 %1, %0 offset:%5\n\t"
               "global_load_lds_dwordx4 %2, %0 offset:%6\n\ts_mov_b64 exec, -1"
               : : "s"(base), "v"(off0), "v"(off1), "s"(lds_tile), "s"(mask), "n"(FIRST * 1024), "n"(FIRST * 1024 + 1024) : "memory", "m0");
}
// One tensor's copies by the WAVES wavefronts of a workgroup, 8 / WAVES pieces each.
template <int WAVES>
struct TileCopy {
  static constexpr int PPW = 8 / WAVES;
  const char* slice;   // the (b,h) slice's first token
  long long snb;       // bytes from one token to the next
  unsigned odd;        // 0: 16-byte aligned rows at a stride that the 32-bit offsets below reach
  unsigned off[4];     // this lane's byte offset in pieces i, i + 4 of its wavefront
  int w, lane;
  __device__ __forceinline__ void init(const bf16_t* x, long long sn, int w_, int lane_) {
    slice = (const char*)x;
    snb = 2 * sn;
    odd = ((unsigned)(uintptr_t)x & 15u) | (unsigned)(snb >> 26);
    w = w_;
    lane = lane_;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * i + (lane >> 4);
      off[i] = (unsigned)((4 * PPW * w + r) * snb) + (((lane & 15) ^ swz(4 * PPW * w + r)) << 4);
    }
  }
  // For copies of several pieces with immediate offsets: piece i reads base3 + off3(i) + 1024 i.
  __device__ __forceinline__ const char* base3(int row0) const { return slice + row0 * snb - 3 * 1024; }
  __device__ __forceinline__ unsigned off3(int i) const { return off[i] + (3 - i) * 1024; }
  __device__ __forceinline__ unsigned dst(unsigned lds_tile) const { return __builtin_amdgcn_readfirstlane(lds_tile + w * PPW * 1024); }
  // Are rows row0 .. row0 + rows - 1 whole, and their copies of the plain kind?  (uniform)
  __device__ __forceinline__ bool plain(int row0, int rows, int N) const { return row0 + rows <= N && odd == 0; }
  // rows row0 .. row0 + 31; rows beyond N come as row N - 1 (their weight is zero) or, if asked for, as zeros
  template <bool ZEROS = false>
  __device__ __forceinline__ void tile(int row0, int N, unsigned lds_tile) const {
    if (__builtin_expect(plain(row0, 32, N), 1)) {
      const char* b = slice + row0 * snb;
#pragma unroll
      for (int i = 0; i < PPW; ++i) copy_piece(i < 4 ? b : b + 16 * snb, off[i & 3], dst(lds_tile) + i * 1024);
    } else {
      tile_any<ZEROS>(row0, N, lds_tile);
    }
  }
  template <bool ZEROS = false>
  __device__ __forceinline__ void tile_any(int row0, int N, unsigned lds_tile) const {
    int ln = lane;
    asm volatile("" : "+v"(ln));            // (nothing of this path is worth a register outside of it)
#pragma unroll 1
    for (int i = 0; i < PPW; ++i) {
      const int r = 4 * (PPW * w + i) + (ln >> 4);
      const char* src = slice + min(row0 + r, N - 1) * snb + (((ln & 15) ^ swz(r)) << 4);
      if (ZEROS && row0 + r >= N) {         // (fewer copies may be under way then than the caller counts: it waits for all of them)
        *(__attribute__((address_space(3))) v4i*)(uintptr_t)(dst(lds_tile) + i * 1024 + ln * 16) = v4i{};
      } else if ((odd & 15u) == 0) {
        copy_piece(src, dst(lds_tile) + i * 1024);
      } else {
        // A contiguous tensor may start at any element.  The asynchronous copies take whole 16-byte units only, an
        // ordinary load takes any address: through a register.  (It has arrived before the next one is requested, so
        // waiting by count errs on the safe side.)
        v4i got;
        __builtin_memcpy(&got, src, 16);
        *(__attribute__((address_space(3))) v4i*)(uintptr_t)(dst(lds_tile) + i * 1024 + ln * 16) = got;
      }
    }
  }
};
// n_op on such a tile: swz_lane_offset once per lane, the step's bits flipped in.
__device__ __forceinline__ int swz_lane_offset(int l32, int hf) { return l32 * 256 + ((hf ^ swz(l32)) << 4); }
__device__ __forceinline__ uint4 n_op_swz(const unsigned char* tile, int lane_off, int ks) {
  return *(const uint4*)(tile + (lane_off ^ (ks << 5)));
}
// t_op on such a tile (the same lane, row and channel assignment).
__device__ __forceinline__ int swz_tr_lane_offset(int lane) {
  const int hf = lane >> 5, row = 4 * hf + ((lane & 15) >> 2), chunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  return row * 256 + ((chunk ^ swz(row)) << 4) + 8 * (lane & 1);
}
__device__ __forceinline__ uint4 t_op_swz(const unsigned char* tile, int tr_off, int ct, int s) {
  union { v4s h[2]; uint4 v; } u;
  u.h[0] = read_tr(tile + 16 * s * 256 + (tr_off ^ (ct << 6)));
  u.h[1] = read_tr(tile + (16 * s + 8) * 256 + (tr_off ^ (ct << 6) ^ (2 << 4)));   // (eight rows on: swz flips bit 1)
  return u.v;
}
// 64 consecutive floats global -> LDS, one per lane.
__device__ __forceinline__ void copy_floats(const float* base, unsigned off, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, %0" : : "s"(base), "v"(off), "s"(lds_addr) : "memory", "m0");
}
// Waits for all but COUNT of this wavefront's copies and for its LDS reads, then meets the workgroup's other wavefronts.
// (SLA_FULL_WAITS: a checking build that waits for all of them, whose results have to be the same bits.)
template <int COUNT>
__device__ __forceinline__ void copies_barrier() {
  static_assert(COUNT < 64, "the counter's range");
#ifdef SLA_FULL_WAITS
  constexpr int KEEP = 0;
#else
  constexpr int KEEP = COUNT;
#endif
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (KEEP & 15) | ((KEEP >> 4) << 14));  // vmcnt(KEEP) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace sla
