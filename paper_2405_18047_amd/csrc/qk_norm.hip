// Norms of query and key heads for gfx950, with the rotary positions in the same pass: y = R(position) (x / rms(x) * g) for every head, g the gains
// of the query or of the key heads; backward-p1 with the gains' gradient left as partial rows for backward-p2; and the serving form,
// which puts the keys and values of new tokens into a cache.
//
//   n = x r, r = 1 / sqrt(mean(x^2) + eps);  z = n g;  y = R z
//   dz = R^T dy;  dn = dz g;  dx = r (dn - n mean(dn n)) = r dn - x r^3 mean(dn x);  dg = sum over tokens and heads of dz n
//
// A unit is two pieces of W columns, of the rotated ones or of the others, half of them apart: half-split positions pair the two, interleaved ones the columns within
// each (W 1: the two columns of a pair).  A group of lanes (a power of two) has one unit each (W 1: up to NU) of one head, so that a head's sums are a few lane
// exchanges, and takes HPT consecutive heads of one kind, which share angles and gains; all of them are loaded before the first is stored, so that
// results may go where the operands came from.
// Bound by memory: 8192 rows of 32 + 8 heads of 128, bf16, half-split, positions given: 33 us forward, 168 MB, 5.1 TB/s; 50 us backward, 252 MB, 5.0 TB/s.
#include "kernels.h"
#include "rows.h"

#include <type_traits>

namespace tbp {

// Columns and angles of a lane's units.
template <typename T, int W, int NU, bool INTERLEAVED>
struct Units {
  static constexpr bool PAIRS = INTERLEAVED && W == 1;      // a pair is the unit's two columns side by side
  int first[NU], second[NU];                       // columns of the two pieces
  bool there[NU], turns[NU];
  float cs[NU][W], sn[NU][W];
  __device__ __forceinline__ Units(const QkNormParams& p, int l) {
    const int rot = p.half / W;
#pragma unroll
    for (int i = 0; i < NU; i++) {
      const int u = l + i * p.lanes;
      there[i] = u < p.units;
      turns[i] = u < rot;
      const int start = turns[i] ? 0 : 2 * p.half, apart = turns[i] ? p.half : p.dh / 2 - p.half, at = (turns[i] ? u : u - rot) * W;
      first[i] = PAIRS ? 2 * u : start + at;
      second[i] = PAIRS ? 2 * u + 1 : start + apart + at;
    }
  }
  __device__ __forceinline__ void angles(const QkNormParams& p, int l, int pos) {
    const bool known = pos >= 0 && pos < p.n_pos;
#pragma unroll
    for (int i = 0; i < NU; i++) {
      if (!turns[i]) continue;
      const float2* const tb = p.table + (known ? (long)pos * p.half : 0);
      const int u = l + i * p.lanes;
      if constexpr (W > 1) {                       // (whole pieces: 16-byte aligned)
#pragma unroll
        for (int k = 0; k < W; k += 2) {
          const f32x4 t = *reinterpret_cast<const f32x4*>(tb + (!INTERLEAVED ? u * W + k : (k < W / 2 ? first[i] : second[i] - W) / 2 + k));
          cs[i][k] = t[0]; sn[i][k] = t[1]; cs[i][k + 1] = t[2]; sn[i][k + 1] = t[3];
        }
      } else {
        cs[i][0] = tb[u].x;
        sn[i][0] = tb[u].y;
      }
      if (!known) {
#pragma unroll
        for (int k = 0; k < W; k++) cs[i][k] = sn[i][k] = __builtin_nanf("");
      }
    }
  }
  // pairs of a unit's 2 W values turned by the angles, or back
  __device__ __forceinline__ void turn(int i, float* v, float sgn) const {
    if (!turns[i]) return;
#pragma unroll
    for (int k = 0; k < W; k++) {
      float& a = v[INTERLEAVED ? 2 * k : k];
      float& b = v[INTERLEAVED ? 2 * k + 1 : W + k];
      const float s = sn[i][k] * sgn, e = a * cs[i][k] - b * s, o = a * s + b * cs[i][k];
      a = e;
      b = o;
    }
  }
};

template <typename T, int W> struct Unit {         // a unit as it lies in memory
  using P = Piece<T, W>;
  typename P::Raw a, b;
  __device__ __forceinline__ void load(const T* p, int first, int second) { a = P::load(p + first); b = P::load(p + second); }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int i = 0; i < W; i++) { v[i] = (float)a.v[i]; v[W + i] = (float)b.v[i]; }
  }
  __device__ __forceinline__ void set(const float* v) {
#pragma unroll
    for (int i = 0; i < W; i++) { a.v[i] = (T)v[i]; b.v[i] = (T)v[W + i]; }
  }
  __device__ __forceinline__ void store(T* p, int first, int second) const { P::store(p + first, a); P::store(p + second, b); }
};

// gains are read over and over: through the caches
template <typename T, int W> __device__ __forceinline__ void load_gain(const T* g, int first, int second, float* v) {
  typedef typename Piece<T, W>::Raw Raw;
  const Raw a = *reinterpret_cast<const Raw*>(g + first), b = *reinterpret_cast<const Raw*>(g + second);
#pragma unroll
  for (int i = 0; i < W; i++) { v[i] = (float)a.v[i]; v[W + i] = (float)b.v[i]; }
}

template <typename T, int W, int NU, int HPT, bool INTERLEAVED, bool APPEND>
__global__ __launch_bounds__(256) void qk_norm_kernel(QkNormParams p) {
  const long at = ((long)blockIdx.x * 256 + threadIdx.x) / p.lanes;
  const int l = (int)threadIdx.x & (p.lanes - 1);
  if (at >= p.items) return;
  const int groups = p.q_groups + (APPEND ? 2 : 1) * p.kv_groups;
  const int of_launch = (int)((unsigned)at / (unsigned)groups), hg = (int)((unsigned)at - (unsigned)of_launch * groups), row = p.row0 + of_launch;
  const int kind = hg < p.q_groups ? 0 : hg < p.q_groups + p.kv_groups ? 1 : 2;      // q, k, v
  const int h0 = (hg - (kind == 0 ? 0 : p.q_groups + (kind == 2 ? p.kv_groups : 0))) * HPT, heads = kind == 0 ? p.q_heads : p.kv_heads;
  const int hn = heads - h0 < HPT ? heads - h0 : HPT;
  const int column = ((kind == 0 ? 0 : p.q_heads + (kind == 2 ? p.kv_heads : 0)) + h0) * p.dh;

  int pos;
  long slot = -1;                                  // (APPEND) row of the caches, or none
  bool idle = false;
  if constexpr (APPEND) {
    const int b = row / p.tokens_new, len = p.lengths[b], ring = p.capacity - p.sinks;
    pos = len - p.tokens_new + (row - b * p.tokens_new);
    idle = pos < 0;
    if (!idle && (pos < p.sinks || pos >= len - ring))        // (a later one of these tokens takes the others' slots over)
      slot = (long)b * p.capacity + (pos < p.sinks ? pos : p.sinks + (pos - p.sinks) % ring);
  } else {
    pos = p.positions ? p.positions[row] : row % p.seq;
  }
  Units<T, W, NU, INTERLEAVED> un(p, l);
  Unit<T, W> x[HPT][NU];
  const T* const src = (const T*)p.x + (long)row * p.ld_x + column;
#pragma unroll
  for (int k = 0; k < HPT; k++)
#pragma unroll
    for (int i = 0; i < NU; i++) if (k < hn && un.there[i]) x[k][i].load(src + (long)k * p.dh, un.first[i], un.second[i]);
  T* dst = (T*)p.y + (long)row * p.ld_y + column;
  if constexpr (APPEND) if (kind > 0) {
    if (slot < 0) return;
    dst = (T*)(kind == 1 ? p.cache_k : p.cache_v) + slot * p.ld_c + (long)h0 * p.dh;
  }
  if (kind < 2) {
    const T* const gain = (const T*)(kind == 0 ? p.gq : p.gk);
    float g[NU][2 * W];
#pragma unroll
    for (int i = 0; i < NU; i++) if (un.there[i]) load_gain<T, W>(gain, un.first[i], un.second[i], g[i]);
    un.angles(p, l, pos);
#pragma unroll
    for (int k = 0; k < HPT; k++) {
      if (k >= hn) break;
      float v[NU][2 * W], ss = 0.f;
#pragma unroll
      for (int i = 0; i < NU; i++) if (un.there[i]) {
        x[k][i].get(v[i]);
#pragma unroll
        for (int c = 0; c < 2 * W; c++) ss += v[i][c] * v[i][c];
      }
      const float r = idle ? 0.f : rsqrtf(group_sum(ss, p.lanes) / (float)p.dh + p.eps);
#pragma unroll
      for (int i = 0; i < NU; i++) if (un.there[i]) {
#pragma unroll
        for (int c = 0; c < 2 * W; c++) v[i][c] = idle ? 0.f : v[i][c] * r * g[i][c];
        if (!idle) un.turn(i, v[i], 1.f);
        x[k][i].set(v[i]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < HPT; k++)
#pragma unroll
    for (int i = 0; i < NU; i++) if (k < hn && un.there[i]) x[k][i].store(dst + (long)k * p.dh, un.first[i], un.second[i]);
}

// backward-p1: the first q_parts workgroups walk (row, query heads) items, the others (row, key heads), and each leaves one partial row of the gains' gradient,
// [2][dh], zeros for the other kind: summed over a lane's items first, then over the lanes of a wave that have the same columns, then over the waves
// in order: the same result every time.
template <typename T, int W, int NU, int HPT, bool INTERLEAVED>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(4))) void qk_norm_p1_kernel(QkNormParams p) {
  extern __shared__ float sums[];                  // [8 waves][dh]
  const int l = (int)threadIdx.x & (p.lanes - 1), per = 512 / p.lanes;
  const bool kind = (int)blockIdx.x >= p.q_parts;
  const int groups = kind ? p.kv_groups : p.q_groups, heads = kind ? p.kv_heads : p.q_heads;
  const int parts = kind ? (int)gridDim.x - p.q_parts : p.q_parts, part = (int)blockIdx.x - (kind ? p.q_parts : 0);
  Units<T, W, NU, INTERLEAVED> un(p, l);
  const T* const gain = (const T*)(kind ? p.gk : p.gq);
  float g[NU][2 * W], dg[NU][2 * W];
#pragma unroll
  for (int i = 0; i < NU; i++) {
    if (un.there[i]) load_gain<T, W>(gain, un.first[i], un.second[i], g[i]);
#pragma unroll
    for (int c = 0; c < 2 * W; c++) dg[i][c] = 0.f;
  }
  const float over = 1.f / (float)p.dh;
  const long items = (long)p.rows * groups;
  for (long at = (long)part * per + threadIdx.x / p.lanes; at < items; at += (long)parts * per) {
    const int row = (int)(at / groups), h0 = (int)(at - (long)row * groups) * HPT;
    const int hn = heads - h0 < HPT ? heads - h0 : HPT;
    const int column = ((kind ? p.q_heads : 0) + h0) * p.dh;
    Unit<T, W> x[HPT][NU], d[HPT][NU];
    const T* const src = (const T*)p.x + (long)row * p.ld_x + column;
    const T* const dsrc = (const T*)p.dy + (long)row * p.ld_dy + column;
#pragma unroll
    for (int k = 0; k < HPT; k++)
#pragma unroll
      for (int i = 0; i < NU; i++) if (k < hn && un.there[i]) {
        x[k][i].load(src + (long)k * p.dh, un.first[i], un.second[i]);
        d[k][i].load(dsrc + (long)k * p.dh, un.first[i], un.second[i]);
      }
    un.angles(p, l, p.positions ? p.positions[row] : row % p.seq);
#pragma unroll
    for (int k = 0; k < HPT; k++) {
      if (k >= hn) break;
      float v[NU][2 * W], dz[NU][2 * W], ss = 0.f, sd = 0.f;
#pragma unroll
      for (int i = 0; i < NU; i++) if (un.there[i]) {
        x[k][i].get(v[i]);
        d[k][i].get(dz[i]);
        un.turn(i, dz[i], -1.f);
#pragma unroll
        for (int c = 0; c < 2 * W; c++) { ss += v[i][c] * v[i][c]; sd += dz[i][c] * g[i][c] * v[i][c]; }
      }
      const float r = rsqrtf(group_sum(ss, p.lanes) * over + p.eps);
      const float back = group_sum(sd, p.lanes) * over * r * r;      // mean(dn x) r^2
#pragma unroll
      for (int i = 0; i < NU; i++) if (un.there[i]) {
        float o[2 * W];
#pragma unroll
        for (int c = 0; c < 2 * W; c++) {
          dg[i][c] += dz[i][c] * (v[i][c] * r);
          o[c] = r * (dz[i][c] * g[i][c] - v[i][c] * back);
        }
        d[k][i].set(o);
      }
    }
    T* const dst = (T*)p.y + (long)row * p.ld_y + column;
#pragma unroll
    for (int k = 0; k < HPT; k++)
#pragma unroll
      for (int i = 0; i < NU; i++) if (k < hn && un.there[i]) d[k][i].store(dst + (long)k * p.dh, un.first[i], un.second[i]);
  }
  const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < NU; i++)
#pragma unroll
    for (int c = 0; c < 2 * W; c++) {
      float s = dg[i][c];
      for (int o = p.lanes; o < 64; o *= 2) s += __shfl_xor(s, o);
      if (lane < p.lanes && un.there[i]) sums[wave * p.dh + (c < W ? un.first[i] + c : un.second[i] + c - W)] = s;
    }
  __syncthreads();
  for (int c = (int)threadIdx.x; c < 2 * p.dh; c += 512) {
    const bool k = c >= p.dh;
    float s = 0.f;
    if (k == kind) {
#pragma unroll
      for (int w = 0; w < 8; w++) s += sums[w * p.dh + (k ? c - p.dh : c)];
    }
    p.partials[(long)blockIdx.x * 2 * p.dh + c] = s;
  }
}

// ------------------------------------------------------------------------------------------ launches
static int lanes_of(int units) {
  int n = 1;
  while (n < units && n < 64) n *= 2;
  return n;
}

// 16-byte pieces, if rotated columns, heads and the starts of all rows go by them; else single elements.
template <typename T>
static bool wide(const QkNormParams& p) {
  constexpr int W = 16 / sizeof(T);
  const uintptr_t bits = (uintptr_t)p.x | (uintptr_t)p.y | (uintptr_t)p.dy | (uintptr_t)p.cache_k | (uintptr_t)p.cache_v |
                         (uintptr_t)p.gq | (uintptr_t)p.gk | (uintptr_t)p.table | (uintptr_t)((p.ld_x | p.ld_y | p.ld_dy | p.ld_c) * sizeof(T));
  return bits % 16 == 0 && p.half % W == 0 && (p.dh - 2 * p.half) % (2 * W) == 0;
}

template <typename T, int W, int NU, int HPT, bool INTERLEAVED, bool APPEND>
static hipError_t launch_fwd(QkNormParams p, hipStream_t s) {
  p.units = p.dh / (2 * W);
  p.lanes = lanes_of(p.units);
  p.q_groups = (p.q_heads + HPT - 1) / HPT;
  p.kv_groups = (p.kv_heads + HPT - 1) / HPT;
  const long groups = p.q_groups + (APPEND ? 2 : 1) * p.kv_groups, most = (1L << 31) / (groups * p.lanes);      // (a launch's threads are counted in 32 bits)
  for (p.row0 = 0; p.row0 < p.rows;) {
    const long n = p.rows - p.row0 < most ? p.rows - p.row0 : most;
    p.items = n * groups;
    hipLaunchKernelGGL((qk_norm_kernel<T, W, NU, HPT, INTERLEAVED, APPEND>), dim3((unsigned)((p.items * p.lanes + 255) / 256)), dim3(256), 0, s, p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    p.row0 += (int)n;
  }
  return hipSuccess;
}

int qk_norm_partial_rows(int rows, int q_heads, int kv_heads, int head_dim) {
  const long n = ((long)rows * ((long)q_heads + kv_heads) * head_dim + 4095) / 4096, least = q_heads && kv_heads ? 2 : 1;
  return (int)(n < least ? least : n < kQkNormPartials ? n : kQkNormPartials);
}

template <typename T, int W, int NU, int HPT, bool INTERLEAVED>
static hipError_t launch_p1(QkNormParams p, hipStream_t s) {
  p.units = p.dh / (2 * W);
  p.lanes = lanes_of(p.units);
  p.q_groups = (p.q_heads + HPT - 1) / HPT;
  p.kv_groups = (p.kv_heads + HPT - 1) / HPT;
  p.n_partials = qk_norm_partial_rows(p.rows, p.q_heads, p.kv_heads, p.dh);
  p.q_parts = p.n_partials;
  if (p.kv_heads) {
    const long share = ((long)p.n_partials * p.q_groups + (p.q_groups + p.kv_groups) / 2) / (p.q_groups + p.kv_groups);
    p.q_parts = !p.q_heads ? 0 : share < 1 ? 1 : share < p.n_partials ? (int)share : p.n_partials - 1;
  }
  hipLaunchKernelGGL((qk_norm_p1_kernel<T, W, NU, HPT, INTERLEAVED>), dim3((unsigned)p.n_partials), dim3(512), 8 * p.dh * sizeof(float), s, p);
  return hipGetLastError();
}

// heads per thread in the forward: four share angles and gains and load more at a time; one, where four leave compute units short of workgroups.  us, one / four, 40 heads of 128,
// bf16: 1024 rows 7.7 / 7.5, 2048 11.0 / 9.1, 8192 32.0 / 32.6; 16 of 64: 8192 rows 11.3 / 8.7; fp32, 40 of 128: 1024 9.7 / 7.9.  In backward-p1 always one: four take 220 registers of
// the 128 that four waves per SIMD have: 8192 rows of 40 heads of 128 70 us for 50.
int qk_norm_heads_per_thread(int dtype, int rows, int q_heads, int kv_heads, int head_dim) {
  const int w = dtype ? 8 : 4;
  return (long)rows * (((long)q_heads + kv_heads + 3) / 4) * (head_dim / (2 * w)) >= 384 * 256 ? 4 : 1;
}

template <typename T, bool APPEND>
static hipError_t forward(const QkNormParams& p, hipStream_t s) {
  constexpr int W = 16 / sizeof(T);
  if (!wide<T>(p)) return p.interleaved ? launch_fwd<T, 1, 4, 1, true, APPEND>(p, s) : launch_fwd<T, 1, 4, 1, false, APPEND>(p, s);
  if (qk_norm_heads_per_thread(sizeof(T) == 2, p.rows, p.q_heads, p.kv_heads, p.dh) == 4) return p.interleaved ? launch_fwd<T, W, 1, 4, true, APPEND>(p, s) : launch_fwd<T, W, 1, 4, false, APPEND>(p, s);
  return p.interleaved ? launch_fwd<T, W, 1, 1, true, APPEND>(p, s) : launch_fwd<T, W, 1, 1, false, APPEND>(p, s);
}

template <typename T>
static hipError_t backward(const QkNormParams& p, hipStream_t s) {
  constexpr int W = 16 / sizeof(T);
  if (!wide<T>(p)) return p.interleaved ? launch_p1<T, 1, 4, 1, true>(p, s) : launch_p1<T, 1, 4, 1, false>(p, s);
  return p.interleaved ? launch_p1<T, W, 1, 1, true>(p, s) : launch_p1<T, W, 1, 1, false>(p, s);
}

hipError_t qk_norm(int dtype, const QkNormParams& p, hipStream_t s) { return dtype ? forward<bf16_t, false>(p, s) : forward<float, false>(p, s); }
hipError_t qk_norm_append(int dtype, const QkNormParams& p, hipStream_t s) { return dtype ? forward<bf16_t, true>(p, s) : forward<float, true>(p, s); }
hipError_t qk_norm_p1(int dtype, const QkNormParams& p, hipStream_t s) { return dtype ? backward<bf16_t>(p, s) : backward<float>(p, s); }

}  // namespace tbp
