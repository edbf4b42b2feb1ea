// What the HBM-bound kernels share: 16-byte accesses unpacked to fp32, and wavefront reductions.
#pragma once
#include "gfx950.h"

namespace tbp {

// ---- 16-byte vector access, unpacked to fp32 ------------------------------------------------------
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  typedef float4 Raw;
  static __device__ __forceinline__ Raw load_raw(const float* p) { return *reinterpret_cast<const float4*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& r, float* v) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
  static __device__ __forceinline__ void load(const float* p, float* v) {
    const float4 r = *reinterpret_cast<const float4*>(p);
    v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w;
  }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <> struct Vec<bf16_t> {
  static constexpr int N = 8;
  typedef u32x4 Raw;
  static __device__ __forceinline__ Raw load_raw(const bf16_t* p) { return *reinterpret_cast<const u32x4*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& r, float* v) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[2 * i] = __uint_as_float(r[i] << 16);
      v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void load(const bf16_t* p, float* v) {
    const u32x4 r = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[2 * i] = __uint_as_float(r[i] << 16);
      v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float* v) {
    typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; i++) o[i] = (bf16_t)v[i];      // round to nearest even
    *reinterpret_cast<bf16x8*>(p) = o;
  }
};

// Wavefront (64-lane) reductions on the data-parallel-primitive path: four in-row steps (quad swaps, half-row and
// row mirrors), then the row totals are chained with row_bcast15 / row_bcast31, which leaves the result in lane 63.
// No LDS traffic and no cross-lane permute unit involved.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_move(float identity, float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, identity),
                                                               __builtin_bit_cast(int, v), CTRL, ROW_MASK, 0xF, false));
}
__device__ __forceinline__ float wave_sum(float v) {
  v += dpp_move<0xB1, 0xF>(0.f, v);     // quad_perm [1,0,3,2]
  v += dpp_move<0x4E, 0xF>(0.f, v);     // quad_perm [2,3,0,1]
  v += dpp_move<0x141, 0xF>(0.f, v);    // row_half_mirror
  v += dpp_move<0x140, 0xF>(0.f, v);    // row_mirror: every lane of a 16-lane row holds the row total
  v += dpp_move<0x142, 0xA>(0.f, v);    // row_bcast15 into rows 1 and 3
  v += dpp_move<0x143, 0xC>(0.f, v);    // row_bcast31 into rows 2 and 3: lane 63 holds the wave total
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  const float ninf = -INFINITY;
  v = fmaxf(v, dpp_move<0xB1, 0xF>(ninf, v));
  v = fmaxf(v, dpp_move<0x4E, 0xF>(ninf, v));
  v = fmaxf(v, dpp_move<0x141, 0xF>(ninf, v));
  v = fmaxf(v, dpp_move<0x140, 0xF>(ninf, v));
  v = fmaxf(v, dpp_move<0x142, 0xA>(ninf, v));
  v = fmaxf(v, dpp_move<0x143, 0xC>(ninf, v));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

}  // namespace tbp
