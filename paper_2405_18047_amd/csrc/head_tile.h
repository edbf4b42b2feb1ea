// LDS images of attention heads (rows of head_dim bf16 values) and the fragments that the matrix instructions read from them,
// shared by the attention kernels.
#pragma once
#include "gfx950.h"

namespace tbp {

// LDS image of `rows` x DH bf16, filled by asynchronous copies (a wave-wide copy writes 1 KiB = 4 or 8 rows).
// The 16-byte granule G of row r sits in slot G ^ swz(r).  swz is a bit permutation of the row index chosen so that
// both access patterns are free of bank conflicts: 16 consecutive rows at one granule (row fragments, ds_read_b128)
// and 4 consecutive rows x 2 adjacent granules (transpose fragments, ds_read_b64_tr_b16).
template <int DH>
struct HeadTile {
  static constexpr int RB = DH * 2, GPRW = DH / 8, RPC = 1024 / RB;
  static __device__ __forceinline__ int swz(int r) {
    if constexpr (DH == 128) return ((r & 3) << 1) | ((r >> 2) & 1) | (r & 8);
    else return (((r >> 1) & 1) << 1) | ((r >> 2) & 1) | (((r >> 3) & 1) << 2);
  }
  static __device__ __forceinline__ int at(int r, int G) { return r * RB + ((G ^ swz(r)) << 4); }
  // Copy plan of lane p of chunk c: tile row and byte offset inside the source row block.
  static __device__ __forceinline__ void plan(int c, int p, long ld, int& row, unsigned& goff) {
    row = RPC * c + p / GPRW;
    const int G = (p % GPRW) ^ swz(row);
    goff = (unsigned)((long)row * ld * 2 + G * 16);
  }
  // The same for an image whose rows are 32 rows of one head after the other: row r of the image is source row 32 (r / 32 / HEADS) + r % 32, head r / 32 % HEADS.
  template <int HEADS> static __device__ __forceinline__ void plan_heads(int c, int p, long ld, int& row, unsigned& goff) {
    plan(c, p, HEADS == 1 ? ld : 0, row, goff);
    if constexpr (HEADS > 1) {
      const int head = row / 32 % HEADS;
      row = 32 * (row / 32 / HEADS) + row % 32;
      goff += (unsigned)((long)row * ld * 2 + head * RB);
    }
  }
  // Per-lane byte offsets of the fragment reads, computed once per kernel (the swizzle makes them non-affine in the
  // k-step, so they are kept in registers; everything else - image, 32-row block, k-step pair - is an immediate).
  //   rows[s]: A-operand fragment of MFMA rows 0..31 of the image, contraction = columns 16 s .. 16 s + 15.
  //   cols[t][0/1]: A-operand fragment of the TRANSPOSED image: MFMA rows = columns 32 t .. 32 t + 31, contraction =
  //            image rows 16 u + {0..3} + 4 (lane / 32) (first read) and 16 u + 8 + {0..3} + 4 (lane / 32) (second):
  //            the accumulator row order, see the file header.  16 u rows further is an immediate too.
  struct Offsets { int rows[DH / 16]; int cols[DH / 32][2]; };
  static __device__ __forceinline__ Offsets offsets(int lane) {
    Offsets o;
#pragma unroll
    for (int s = 0; s < DH / 16; s++) o.rows[s] = at(lane & 31, 2 * s + (lane >> 5));
    const int i = lane & 15, q = (lane >> 4) & 1, g = lane >> 5;
    const int r = 4 * g + (i >> 2);
#pragma unroll
    for (int t = 0; t < DH / 32; t++) {
      const int G = 2 * (2 * t + q) + ((i & 3) >> 1);
      o.cols[t][0] = at(r, G) + 8 * (i & 1);
      o.cols[t][1] = at(r + 8, G) + 8 * (i & 1);
    }
    return o;
  }
  static __device__ __forceinline__ bf16x8 rows_frag(lds_u8* img, const Offsets& o, int r0, int s) {   // r0 % 16 == 0
    return *reinterpret_cast<LDS_AS const bf16x8*>(img + o.rows[s] + r0 * RB);
  }
  static __device__ __forceinline__ bf16x8 cols_frag(lds_u8* img, const Offsets& o, int r0, int u, int t) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_AS s16x4*>(img + o.cols[t][0] + (r0 + 16 * u) * RB));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_AS s16x4*>(img + o.cols[t][1] + (r0 + 16 * u) * RB));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

__device__ __forceinline__ float xor32(float v) { return __shfl_xor(v, 32, 64); }

__device__ __forceinline__ bf16x8 pack8(const f32x16& c, int u) {
  bf16x8 b;
#pragma unroll
  for (int t = 0; t < 8; t++) b[t] = (bf16_t)c[8 * u + t];
  return b;
}

}  // namespace tbp
