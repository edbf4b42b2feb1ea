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

// W elements as they lie in memory.  Each is touched once: 16-byte pieces go past the caches' retention (nontemporal), which takes the
// [8192, 5120] case from 38.5 us to 32.6, fp32 from 61.0 to 54.6.
template <typename T, int W> struct Piece {
  struct alignas(sizeof(T) * W) Raw { T v[W]; };
  static __device__ __forceinline__ Raw load(const T* p) {
    if constexpr (sizeof(Raw) == 16) return __builtin_bit_cast(Raw, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
    else return *reinterpret_cast<const Raw*>(p);
  }
  static __device__ __forceinline__ void store(T* p, const Raw& r) {
    if constexpr (sizeof(Raw) == 16) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), reinterpret_cast<u32x4*>(p));
    else *reinterpret_cast<Raw*>(p) = r;
  }
};

// A thread owns one unit of a row's heads and applies the cosines and sines that it holds to HPT consecutive heads.  A unit is
//   INSIDE  W columns that hold whole pairs (interleaved);
//   ACROSS  W columns whose partners are another lane's (half-split heads of 1, 2, 4 .. 64 pieces): a head is then read and written in one piece;
//   BESIDE  W columns and the W columns that they are paired with.
// Behind a head's rotated units follow those of W columns that are passed on.  All heads of a thread are loaded before the first is stored: x
// and y may be the same memory, and a load must not wait for the store before it.
// APPEND: heads are q | k | v; a row is token i of the tokens_new new ones of sequence b, at position lengths[b] - tokens_new + i.  q goes
// to y, k and v to the token's slot of the cache.
// Bound by memory: the 40 heads of 128 of 8192 rows, bf16, out of rows of 6144 columns, 168 MB read and written: 30 us, 5.6 TB/s (part of it from the
// memory-side cache).  A token's heads (16 rows of 20 heads of 64, 84 KB) 3.3 us, as long as a launch takes.
enum RotaryUnit { INSIDE, ACROSS, BESIDE };
template <typename T, int W, int HPT, int UNIT, bool APPEND>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  using P = Piece<T, W>;
  typedef typename P::Raw Raw;
  const long item = (long)blockIdx.x * 256 + threadIdx.x;
  if (item >= p.items) return;
  const unsigned grp = (unsigned)item / (unsigned)p.units;
  const int u = (int)((unsigned)item - grp * (unsigned)p.units);
  const int of_launch = (int)(grp / (unsigned)p.groups), hg = (int)(grp - (unsigned)of_launch * p.groups), row = p.row0 + of_launch;
  const int rot_units = UNIT == BESIDE ? p.half / W : 2 * p.half / W;
  const int partner = p.interleaved ? 1 : p.half;            // (BESIDE; interleaved: W is 1)
  const bool rotates = u < rot_units;
  const int col = !rotates ? 2 * p.half + (u - rot_units) * W : p.interleaved && W == 1 ? 2 * u : u * W;

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
  const int h0 = hg * HPT, hn = p.heads - h0 < HPT ? p.heads - h0 : HPT;
  const T* const src = (const T*)p.x + (long)row * p.ld_x + (long)h0 * p.dh + col;
  Raw a[HPT], c[UNIT == INSIDE ? 1 : HPT];
#pragma unroll
  for (int k = 0; k < HPT; k++) {
    if (k >= hn) break;
    a[k] = P::load(src + (long)k * p.dh);
    if constexpr (UNIT == BESIDE) if (rotates) c[k] = P::load(src + (long)k * p.dh + partner);
  }
  constexpr int NA = UNIT == INSIDE ? W / 2 : W;   // angles of a unit
  const int across = UNIT == ACROSS ? p.half / W : 0;
  const bool upper = UNIT == ACROSS && u >= across;          // the unit holds its pairs' second columns
  float cs[NA], sn[NA];
  if (rotates) {
    const bool known = pos >= 0 && pos < p.n_pos;  // (idle: not used)
    const float2* const tb = p.table + (known ? (long)pos * p.half + (upper ? u - across : u) * NA : 0);
#pragma unroll
    for (int i = 0; i < NA; i++) {
      const float2 t = tb[i];
      cs[i] = known ? t.x : __builtin_nanf("");
      sn[i] = known ? t.y * p.sgn : __builtin_nanf("");
    }
  }
  if constexpr (UNIT == ACROSS) {
    constexpr int WORDS = (int)sizeof(Raw) / 4;
    struct Words { uint32_t v[WORDS]; };
    const int lane = (int)(threadIdx.x & 63), other = rotates ? (upper ? lane - across : lane + across) : lane;
#pragma unroll
    for (int k = 0; k < HPT; k++) {
      if (k >= hn) break;
      Words w = __builtin_bit_cast(Words, a[k]);
#pragma unroll
      for (int i = 0; i < WORDS; i++) w.v[i] = __shfl(w.v[i], other);
      c[k] = __builtin_bit_cast(Raw, w);
    }
  }
#pragma unroll
  for (int k = 0; k < HPT; k++) {
    if (k >= hn) break;
    const int h = h0 + k;
    T* dst = (T*)p.y + (long)row * p.ld_y + (long)h * p.dh + col;
    bool turn = rotates;
    if constexpr (APPEND) {
      if (h >= p.q_heads) {
        if (slot < 0) continue;
        const bool is_v = h >= p.q_heads + p.kv_heads;
        turn = rotates && !is_v;
        dst = (T*)(is_v ? p.cache_v : p.cache_k) + slot * p.ld_c + (long)(h - p.q_heads - (is_v ? p.kv_heads : 0)) * p.dh + col;
      } else if (idle) {
        turn = false;
#pragma unroll
        for (int i = 0; i < W; i++) { a[k].v[i] = (T)0.f; if constexpr (UNIT == BESIDE) c[k].v[i] = (T)0.f; }
      }
    }
    if (turn) {
      if constexpr (UNIT == INSIDE) {
#pragma unroll
        for (int i = 0; i < NA; i++) {
          const float e = (float)a[k].v[2 * i], o = (float)a[k].v[2 * i + 1];
          a[k].v[2 * i] = (T)(e * cs[i] - o * sn[i]);
          a[k].v[2 * i + 1] = (T)(e * sn[i] + o * cs[i]);
        }
      } else if constexpr (UNIT == ACROSS) {
#pragma unroll
        for (int i = 0; i < W; i++) a[k].v[i] = (T)((float)a[k].v[i] * cs[i] + (float)c[k].v[i] * (upper ? sn[i] : -sn[i]));
      } else {
#pragma unroll
        for (int i = 0; i < W; i++) {
          const float e = (float)a[k].v[i], o = (float)c[k].v[i];
          a[k].v[i] = (T)(e * cs[i] - o * sn[i]);
          c[k].v[i] = (T)(e * sn[i] + o * cs[i]);
        }
      }
    }
    P::store(dst, a[k]);
    if constexpr (UNIT == BESIDE) if (rotates) P::store(dst + partner, c[k]);
  }
}

hipError_t rotary_table(int n_pos, int rot_dim, float base, const RotaryScale& sc, float2* table, hipStream_t s) {
  const long n = (long)n_pos * (rot_dim / 2);
  hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, n, rot_dim / 2, (double)base, sc.kind,
                     (double)sc.factor, (double)sc.low, (double)sc.high, (double)sc.original, (double)sc.magnitude, table);
  return hipGetLastError();
}

template <typename T, int W, int UNIT, bool APPEND>
static hipError_t launch_w(RotaryParams p, hipStream_t s) {
  const int rot_units = UNIT == BESIDE ? p.half / W : 2 * p.half / W;
  p.units = rot_units + (p.dh - 2 * p.half) / W;
  auto run = [&](auto hpt) {
    constexpr int HPT = decltype(hpt)::value;
    p.groups = (p.heads + HPT - 1) / HPT;
    const long per_row = (long)p.groups * p.units, most = (1L << 31) / per_row;      // (a launch's threads are counted in 32 bits)
    for (p.row0 = 0; p.row0 < p.rows;) {
      const long n = p.rows - p.row0 < most ? p.rows - p.row0 : most;
      p.items = n * per_row;
      hipLaunchKernelGGL((rotary_kernel<T, W, HPT, UNIT, APPEND>), dim3((unsigned)((p.items + 255) / 256)), dim3(256), 0, s, p);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      p.row0 += (int)n;
    }
    return hipSuccess;
  };
  // heads per thread: four read the table less and load more at a time; one, where four leave fewer than 3 workgroups to two compute units.  us, one /
  // four heads, 40 heads of 128, bf16, half-split: 256 rows 3.9 / 4.1, 512 5.1 / 4.8, 1024 9.0 / 5.7, 8192 41.0 / 30.1; interleaved 3.4 / 3.7, 4.3 / 4.2, 7.5 / 5.2,
  // 37.6 / 28.2; fp32 4.3 / 4.2, 7.4 / 5.2, 11.6 / 7.5, 70.3 / 54.0; 12 heads of 64, bf16: 2048 rows 4.1 / 4.2, 4096 5.9 / 4.9, 8192 10.4 / 5.9
  if ((long)p.rows * ((p.heads + 3) / 4) * p.units >= 384 * 256) return run(std::integral_constant<int, 4>{});
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
  auto run = [&](auto width) {
    constexpr int W = decltype(width)::value;
    if constexpr (W > 1) if (p.interleaved) return launch_w<T, W, INSIDE, APPEND>(p, s);
    // ACROSS where it can be: us, across / beside, four heads a thread each: 40 heads of 128, bf16, 1024 rows 5.7 / 6.0, 8192 30.1 / 29.7, half of the columns turned
    // 30.6 / 33.0, fp32 54.0 / 55.4; 12 heads of 64, 8192 rows 5.9 / 7.9, 32768 19.7 / 24.4.  Interleaved pairs, pieces that hold them / column by column: 8192 rows
    // of 40 heads 28.2 / 52.5, fp32 53.6 / 68.1
    const int pieces = p.dh / W;
    if constexpr (W * sizeof(T) >= 4) if (!p.interleaved && pieces <= 64 && (pieces & (pieces - 1)) == 0) return launch_w<T, W, ACROSS, APPEND>(p, s);
    return launch_w<T, W, BESIDE, APPEND>(p, s);
  };
  if constexpr (sizeof(T) == 2) if (w >= 8) return run(std::integral_constant<int, 8>{});
  if (w >= 4) return run(std::integral_constant<int, 4>{});
  if (w >= 2) return run(std::integral_constant<int, 2>{});
  return run(std::integral_constant<int, 1>{});
}

hipError_t rotary(int dtype, const RotaryParams& p, hipStream_t s) { return dtype ? launch_t<bf16_t, false>(p, s) : launch_t<float, false>(p, s); }
hipError_t rotary_append(int dtype, const RotaryParams& p, hipStream_t s) { return dtype ? launch_t<bf16_t, true>(p, s) : launch_t<float, true>(p, s); }

}  // namespace tbp
