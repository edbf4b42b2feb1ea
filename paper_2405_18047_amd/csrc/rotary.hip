// Rotary positions for gfx950: pairs (i, i + r/2) or (2i, 2i + 1) in the first r columns of every head, angles from a table that
// may be scaled for contexts longer than the model was trained on, positions given or restarting per sequence; and the serving
// form, which rotates new tokens and puts their keys and values into a cache.
#include "kernels.h"
#include "rows.h"

#include <type_traits>

namespace tbp {

// table[p][i] = m (cos, sin)(p theta_i), evaluated in fp64: at 100 000 positions the angle needs 17 bits before the point.
__global__ __launch_bounds__(256) void rotary_table_kernel(long n, int half, double base, int scaling, double factor, double low,
                                                           double high, double original, double magnitude, float2* __restrict__ table) {
  const long idx = (long)blockIdx.x * 256 + threadIdx.x;
  if (idx >= n) return;
  const long p = idx / half;
  const int i = (int)(idx - p * half);
  const double inv = -(double)i / (double)half;
  double theta = pow(base, inv);
  if (scaling == ROTARY_LINEAR) theta /= factor;
  if (scaling == ROTARY_BASE) theta = pow(base * pow(factor, (double)half / (double)(half - 1)), inv);      // r / (r - 2), r = 2 half
  if (scaling == ROTARY_RAMP) {
    const double turns = original * theta * 0.15915494309189535;       // of the pair over the original context
    double keep = (turns - low) / (high - low);
    keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
    theta = theta * ((1 - keep) / factor + keep);
  }
  double s, c;
  sincos((double)p * theta, &s, &c);
  table[idx] = make_float2((float)(magnitude * c), (float)(magnitude * s));
}

// ---- W elements, unpacked to fp32 ---------------------------------------------------------------------
template <typename T, int W> struct Piece {
  struct alignas(sizeof(T) * W) Raw { T v[W]; };
  static __device__ __forceinline__ void load(const T* p, float* v) {
    const Raw r = *reinterpret_cast<const Raw*>(p);
#pragma unroll
    for (int i = 0; i < W; i++) v[i] = (float)r.v[i];
  }
  static __device__ __forceinline__ void store(T* p, const float* v) {
    Raw r;
#pragma unroll
    for (int i = 0; i < W; i++) r.v[i] = (T)v[i];
    *reinterpret_cast<Raw*>(p) = r;
  }
};

// A thread owns one unit of W columns of a row's heads (with the W columns they are paired with, half-split) and applies the
// cosines and sines that it holds to HPT consecutive heads.  Units of a head: half / W (half-split) or 2 half / W (interleaved) that
// rotate, then (dh - 2 half) / W that are passed on.
// APPEND: heads are q | k | v; a row is token i of the tokens_new new ones of sequence b, at position lengths[b] - tokens_new + i.  q goes
// to y, k and v to the token's slot of the cache.
template <typename T, int W, int HPT, bool APPEND>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  const long item = (long)blockIdx.x * 256 + threadIdx.x;
  if (item >= p.items) return;
  const unsigned grp = (unsigned)(item / p.units);
  const int u = (int)(item - (long)grp * p.units);
  const int row = (int)(grp / (unsigned)p.groups), hg = (int)(grp - (unsigned)row * p.groups);
  const T* const x = (const T*)p.x;
  T* const y = (T*)p.y;
  const bool inside = p.interleaved && W > 1;      // a unit holds whole pairs; otherwise two pieces of W columns are paired
  const int rot_units = inside ? 2 * p.half / W : p.half / W;
  const int partner = p.interleaved ? 1 : p.half;
  const bool rotates = u < rot_units;
  const int col = !rotates ? 2 * p.half + (u - rot_units) * W : p.interleaved && W == 1 ? 2 * u : u * W;

  int pos, b = 0;
  long slot = -1;                                  // (APPEND) row of the caches, or none
  bool idle = false;
  if constexpr (APPEND) {
    b = row / p.tokens_new;
    const int len = p.lengths[b];
    pos = len - p.tokens_new + (row - b * p.tokens_new);
    idle = pos < 0;
    const int ring = p.capacity - p.sinks;
    if (!idle && (pos < p.sinks || pos >= len - ring))        // (a later one of these tokens takes the others' slots over)
      slot = (long)b * p.capacity + (pos < p.sinks ? pos : p.sinks + (pos - p.sinks) % ring);
  } else {
    pos = p.positions ? p.positions[row] : row % p.seq;
  }
  constexpr int PW = W == 1 ? 1 : W / 2;           // pairs of an interleaved unit
  float cs[W], sn[W];
  if (rotates && !idle) {
    const bool known = pos >= 0 && pos < p.n_pos;
    const float2* const tb = p.table + (known ? (long)pos * p.half + (inside ? u * PW : u * W) : 0);
#pragma unroll
    for (int i = 0; i < W; i++) {
      if (i < (inside ? PW : W)) {
        const float2 t = tb[i];
        cs[i] = known ? t.x : __builtin_nanf("");
        sn[i] = known ? t.y * p.sgn : __builtin_nanf("");
      }
    }
  }
  const int h0 = hg * HPT, hn = p.heads - h0 < HPT ? p.heads - h0 : HPT;
#pragma unroll 4
  for (int k = 0; k < hn; k++) {
    const int h = h0 + k;
    const T* const src = x + (long)row * p.ld_x + (long)h * p.dh + col;
    T* dst = y + (long)row * p.ld_y + (long)h * p.dh + col;
    bool turn = rotates;
    if constexpr (APPEND) {
      if (h >= p.q_heads) {
        const bool is_v = h >= p.q_heads + p.kv_heads;
        if (slot < 0) continue;
        turn = rotates && !is_v;
        dst = (T*)(is_v ? p.cache_v : p.cache_k) + slot * p.ld_c + (long)(h - p.q_heads - (is_v ? p.kv_heads : 0)) * p.dh + col;
      } else if (idle) {
        float z[W];
#pragma unroll
        for (int i = 0; i < W; i++) z[i] = 0.f;
        Piece<T, W>::store(dst, z);
        if (rotates && !inside) Piece<T, W>::store(dst + partner, z);
        continue;
      }
    }
    float a[W];
    Piece<T, W>::load(src, a);
    if (rotates && !inside) {
      float c[W], ya[W], yc[W];
      Piece<T, W>::load(src + partner, c);
#pragma unroll
      for (int i = 0; i < W; i++) {
        ya[i] = turn ? a[i] * cs[i] - c[i] * sn[i] : a[i];
        yc[i] = turn ? a[i] * sn[i] + c[i] * cs[i] : c[i];
      }
      Piece<T, W>::store(dst, ya);
      Piece<T, W>::store(dst + partner, yc);
    } else {
      if constexpr (W > 1) {
        if (turn) {
#pragma unroll
          for (int i = 0; i < PW; i++) {
            const float e = a[2 * i], o = a[2 * i + 1];
            a[2 * i] = e * cs[i] - o * sn[i];
            a[2 * i + 1] = e * sn[i] + o * cs[i];
          }
        }
      }
      if (rotates || dst != src) Piece<T, W>::store(dst, a);
    }
  }
}

hipError_t rotary_table(int n_pos, int rot_dim, float base, const RotaryScale& sc, float2* table, hipStream_t s) {
  const long n = (long)n_pos * (rot_dim / 2);
  hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, n, rot_dim / 2, (double)base, sc.kind,
                     (double)sc.factor, (double)sc.low, (double)sc.high, (double)sc.original, (double)sc.magnitude, table);
  return hipGetLastError();
}

template <typename T, int W, bool APPEND>
static hipError_t launch_w(RotaryParams p, hipStream_t s) {
  const int rot_units = p.interleaved && W > 1 ? 2 * p.half / W : p.half / W;
  p.units = rot_units + (p.dh - 2 * p.half) / W;
  // heads per thread: 8 read the table least; fewer, down to one, until there are 4 workgroups per compute unit
  auto run = [&](auto hpt) {
    constexpr int HPT = decltype(hpt)::value;
    p.groups = (p.heads + HPT - 1) / HPT;
    p.items = (long)p.rows * p.groups * p.units;
    hipLaunchKernelGGL((rotary_kernel<T, W, HPT, APPEND>), dim3((unsigned)((p.items + 255) / 256)), dim3(256), 0, s, p);
    return hipGetLastError();
  };
  if ((long)p.rows * ((p.heads + 7) / 8) * p.units >= 4 * 256 * 256) return run(std::integral_constant<int, 8>{});
  return run(std::integral_constant<int, 1>{});
}

template <typename T, bool APPEND>
static hipError_t launch_t(const RotaryParams& p, hipStream_t s) {
  // the widest pieces (16 bytes at most) that divide heads and rotated columns and that every row's start is aligned to
  const long unit = p.interleaved ? 2 * (long)p.half : p.half;
  uintptr_t bits = (uintptr_t)p.x | (uintptr_t)p.y | (uintptr_t)(p.ld_x * sizeof(T)) | (uintptr_t)(p.ld_y * sizeof(T)) |
                   (uintptr_t)(unit * sizeof(T)) | (uintptr_t)(p.dh * sizeof(T)) | (uintptr_t)p.cache_k | (uintptr_t)p.cache_v |
                   (uintptr_t)(p.ld_c * sizeof(T));
  const int w = (int)((bits & -bits) > 16 || bits == 0 ? 16 : (bits & -bits)) / (int)sizeof(T);
  if constexpr (sizeof(T) == 2) if (w >= 8) return launch_w<T, 8, APPEND>(p, s);
  if (w >= 4) return launch_w<T, 4, APPEND>(p, s);
  if (w >= 2) return launch_w<T, 2, APPEND>(p, s);
  return launch_w<T, 1, APPEND>(p, s);
}

hipError_t rotary(int dtype, const RotaryParams& p, hipStream_t s) { return dtype ? launch_t<bf16_t, false>(p, s) : launch_t<float, false>(p, s); }
hipError_t rotary_append(int dtype, const RotaryParams& p, hipStream_t s) { return dtype ? launch_t<bf16_t, true>(p, s) : launch_t<float, true>(p, s); }

}  // namespace tbp
