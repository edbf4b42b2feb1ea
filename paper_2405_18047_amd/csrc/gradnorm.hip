// The norm over many gradient tensors, and the gradients clipped to it, for gfx950.  Sums of squares are fp64 throughout (the two
// instructions per element that this costs run at a tenth of the rate that memory delivers elements at): no square of a finite
// gradient overflows, and the norm does not depend on how large its tensors are.
// The sums of the workgroups lie side by side in a workspace; every workgroup of the clipping launch adds them up for itself, in order.
// Bound by memory, which gradients cross twice: the factor depends on all of them, and they are more than the caches hold.  405 M of them in fp32
// (1.62 GB) 240 us for the norm, 6.8 TB/s, and 445 us clipped into bf16, 5.5 TB/s; 0.8 M of them, in the caches, 3.8 + 4.5 us, two launches.
// Long lists pay for a launch of each pass per 96 tensors, and every clipping workgroup for all of the sums: 400 M elements in 12 tensors 670 us, in 96 687, in 291 742,
// in 1000 1043; 10 M in 12 22.2, in 291 50.9, in 1000 122.
#include "kernels.h"
#include "rows.h"

#include <type_traits>

namespace tbp {

// Elements that a workgroup takes at a time: 8192, of lists of up to 16 M elements 4096 (clipping 0.8 M 9.3 / 8.3 us, 0.4 M 9.2 / 8.3; 25 M 63.4 /
// 62.5; 405 M 708 / 717).
constexpr int kPiece = 8192, kSmallPiece = 4096;
constexpr int64_t kSmallList = 16 << 20;
// The norm of a list of more than this reads it past the caches: the clipping launch that follows finds nothing of it there anyway.  us, kept / past,
// the norm, and with clipping into bf16: 1.6 GB 265 / 238 and 709 / 682, 810 MB 143 / 127 and 362 / 347, 405 MB 76.4 / 69.4 and 224 / 218; of
// 202 MB, which the memory-side cache keeps, 43.8 / 39.6, but 91 / 98 with clipping.
constexpr int64_t kStreamedBytes = (int64_t)384 << 20;

// A list's tensors, or some of them, cut into pieces; of CAP tensors at most.  The table is copied with every launch: up to 16 tensors take one for 16
// (1, 6, 12 tensors of 4096 elements, us a call one after another: tables for 96 8.6, 8.7, 8.8, for 16 8.1, 8.3, 8.3).
template <int CAP> struct GradTable {
  static constexpr int kCap = CAP;
  int n, pieces, piece;                              // tensors, their pieces, elements of a piece
  const void* src[CAP]; void* dst[CAP];
  int64_t count[CAP];
  int first[CAP];                                    // the tensor's first piece
};

// Accesses of 16 bytes that are not to be kept in the caches.
template <typename T> __device__ __forceinline__ void load_past(const T* p, float* v) {
  Vec<T>::unpack(__builtin_bit_cast(typename Vec<T>::Raw, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p))), v);
}
__device__ __forceinline__ void store_past(float* p, const float* v) {
  const u32x4 r{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  __builtin_nontemporal_store(r, reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ void store_past(bf16_t* p, const float* v) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; i++) r[i] = (bf16_t)v[i];
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), reinterpret_cast<u32x4*>(p));
}

__device__ __forceinline__ double block_sum(double v) {        // of 256 threads, the same in all, order fixed
  __shared__ double red[4];
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// The tensor that piece i of the list lies in.
template <int CAP>
__device__ __forceinline__ int tensor_of(const GradTable<CAP>& t, int i) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= i) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <typename T, bool PAST, int CAP>
__global__ __launch_bounds__(256) void grad_sumsq_kernel(GradTable<CAP> t, double* __restrict__ sums) {
  constexpr int N = Vec<T>::N;
  double acc = 0.0;
  for (int i = blockIdx.x; i < t.pieces; i += gridDim.x) {
    const int k = tensor_of(t, i);
    const long at = (long)(i - t.first[k]) * t.piece, left = t.count[k] - at;
    const T* const g = (const T*)t.src[k] + at;
    const int n = left < t.piece ? (int)left : t.piece;
    if ((uintptr_t)g % 16 == 0) {
#pragma unroll 4
      for (int j = threadIdx.x * N; j + N <= n; j += 256 * N) {
        float v[N];
        if constexpr (PAST) load_past<T>(g + j, v); else Vec<T>::load(g + j, v);
#pragma unroll
        for (int e = 0; e < N; e++) acc += (double)v[e] * (double)v[e];
      }
      for (int j = n / N * N + threadIdx.x; j < n; j += 256) acc += (double)(float)g[j] * (double)(float)g[j];
    } else {
      for (int j = threadIdx.x; j < n; j += 256) acc += (double)(float)g[j] * (double)(float)g[j];
    }
  }
  acc = block_sum(acc);
  if (threadIdx.x == 0) sums[blockIdx.x] = acc;
}

__global__ __launch_bounds__(256) void grad_sum_kernel(const double* __restrict__ sums, int n, double* __restrict__ out) {
  double acc = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) acc += sums[i];
  acc = block_sum(acc);
  if (threadIdx.x == 0) *out = acc;
}

template <typename T, typename O, int CAP>
__global__ __launch_bounds__(256) void grad_clip_kernel(GradTable<CAP> t, const double* __restrict__ sums, int n_sums, float max_norm, float* __restrict__ norm_out) {
  constexpr int N = Vec<T>::N;
  double acc = 0.0;
  for (int i = threadIdx.x; i < n_sums; i += 256) acc += sums[i];
  const double norm = sqrt(block_sum(acc));
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const bool clips = norm > (double)max_norm && norm < __builtin_inf();
  const float c = clips ? (float)((double)max_norm / norm) : 1.f;
  for (int i = blockIdx.x; i < t.pieces; i += gridDim.x) {
    const int k = tensor_of(t, i);
    if (!clips && (const void*)t.src[k] == t.dst[k]) continue;         // in place, and nothing changes
    const long at = (long)(i - t.first[k]) * t.piece, left = t.count[k] - at;
    const T* const g = (const T*)t.src[k] + at;
    O* const o = (O*)t.dst[k] + at;
    const int n = left < t.piece ? (int)left : t.piece;
    int done = 0;
    if ((uintptr_t)g % 16 == 0 && (uintptr_t)o % 16 == 0) {
#pragma unroll 4
      for (int j = threadIdx.x * 8; j + 8 <= n; j += 256 * 8) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; e += N) Vec<T>::load(g + j + e, v + e);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] *= c;
#pragma unroll
        for (int e = 0; e < 8; e += Vec<O>::N) store_past(o + j + e, v + e);
      }
      done = n / 8 * 8;
    }
    for (int j = done + threadIdx.x; j < n; j += 256) o[j] = (O)((float)g[j] * c);
  }
}

// Walks the list in tables: body(table, workgroups, sums before it).
template <typename F>
static hipError_t tables(int n, const void* const* src, void* const* dst, const int64_t* counts, F body) {
  int sums = 0, i = 0;
  int64_t all = 0;
  for (int k = 0; k < n; k++) all += counts[k];
  const int piece = all <= kSmallList ? kSmallPiece : kPiece;
  auto fill = [&](auto& t) {
    t.n = t.pieces = 0;
    t.piece = piece;
    for (; i < n && t.n < t.kCap; i++) {
      if (counts[i] == 0) continue;
      const int64_t pieces = (counts[i] + piece - 1) / piece;
      if (t.pieces + pieces > (1 << 30)) break;
      t.src[t.n] = src[i]; t.dst[t.n] = dst ? dst[i] : nullptr; t.count[t.n] = counts[i]; t.first[t.n] = t.pieces;
      t.pieces += (int)pieces;
      t.n++;
    }
    if (t.n == 0) return hipSuccess;
    const int grid = t.pieces < kGradSums ? t.pieces : kGradSums, before = sums;
    sums += grid;
    return body(t, grid, before);
  };
  while (i < n) {
    hipError_t e;
    if (n - i <= 16) { GradTable<16> t; e = fill(t); }
    else { GradTable<kGradTable> t; e = fill(t); }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t grad_sumsq(int dtype, int n, const void* const* grads, const int64_t* counts, double* sums, int* n_sums, hipStream_t s) {
  *n_sums = 0;
  int64_t bytes = 0;
  for (int i = 0; i < n; i++) bytes += counts[i] * (dtype ? 2 : 4);
  const bool past = bytes > kStreamedBytes;
  return tables(n, grads, nullptr, counts, [&](const auto& t, int grid, int before) {
    constexpr int CAP = std::decay_t<decltype(t)>::kCap;
    auto kern = dtype ? (past ? grad_sumsq_kernel<bf16_t, true, CAP> : grad_sumsq_kernel<bf16_t, false, CAP>)
                      : (past ? grad_sumsq_kernel<float, true, CAP> : grad_sumsq_kernel<float, false, CAP>);
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), 0, s, t, sums + before);
    *n_sums = before + grid;
    return hipGetLastError();
  });
}

hipError_t grad_sum(const double* sums, int n, double* out, hipStream_t s) {
  hipLaunchKernelGGL(grad_sum_kernel, dim3(1), dim3(256), 0, s, sums, n, out);
  return hipGetLastError();
}

hipError_t grad_clip(int dtype, int out_dtype, int n, const void* const* grads, void* const* outs, const int64_t* counts,
                     const double* sums, int n_sums, float max_norm, float* norm, hipStream_t s) {
  bool first = true;
  const hipError_t e = tables(n, grads, outs, counts, [&](const auto& t, int grid, int) {
    constexpr int CAP = std::decay_t<decltype(t)>::kCap;
    auto kern = dtype ? (out_dtype ? grad_clip_kernel<bf16_t, bf16_t, CAP> : grad_clip_kernel<bf16_t, float, CAP>)
                      : (out_dtype ? grad_clip_kernel<float, bf16_t, CAP> : grad_clip_kernel<float, float, CAP>);
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), 0, s, t, sums, n_sums, max_norm, first ? norm : nullptr);
    first = false;
    return hipGetLastError();
  });
  if (e != hipSuccess || !first) return e;
  GradTable<16> none;                                           // nothing to clip: the norm alone
  none.n = none.pieces = 0;
  hipLaunchKernelGGL((grad_clip_kernel<float, float, 16>), dim3(1), dim3(256), 0, s, none, sums, n_sums, max_norm, norm);
  return hipGetLastError();
}

}  // namespace tbp
