// The norm over many gradient tensors, and the gradients clipped to it, for gfx950.  Sums of squares are fp64 throughout (the two
// instructions per element that this costs run at a tenth of the rate that memory delivers elements at): no square of a finite
// gradient overflows, and the norm does not depend on how large its tensors are.
// The sums of the workgroups lie side by side in a workspace; every workgroup of the clipping launch adds them up for itself, in order.
#include "kernels.h"
#include "rows.h"

namespace tbp {

constexpr int kPiece = 8192;           // elements that a workgroup takes at a time

__device__ __forceinline__ double block_sum(double v) {        // of 256 threads, the same in all, order fixed
  __shared__ double red[4];
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// The tensor that piece i of the list lies in.
__device__ __forceinline__ int tensor_of(const GradTable& t, int i) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= i) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <typename T>
__global__ __launch_bounds__(256) void grad_sumsq_kernel(GradTable t, double* __restrict__ sums) {
  constexpr int N = Vec<T>::N;
  double acc = 0.0;
  for (int i = blockIdx.x; i < t.pieces; i += gridDim.x) {
    const int k = tensor_of(t, i);
    const long at = (long)(i - t.first[k]) * kPiece, left = t.count[k] - at;
    const T* const g = (const T*)t.src[k] + at;
    const int n = left < kPiece ? (int)left : kPiece;
    if ((uintptr_t)g % 16 == 0) {
#pragma unroll 4
      for (int j = threadIdx.x * N; j + N <= n; j += 256 * N) {
        float v[N];
        Vec<T>::load(g + j, v);
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

template <typename T, typename O>
__global__ __launch_bounds__(256) void grad_clip_kernel(GradTable t, const double* __restrict__ sums, int n_sums, float max_norm, float* __restrict__ norm_out) {
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
    const long at = (long)(i - t.first[k]) * kPiece, left = t.count[k] - at;
    const T* const g = (const T*)t.src[k] + at;
    O* const o = (O*)t.dst[k] + at;
    const int n = left < kPiece ? (int)left : kPiece;
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
        for (int e = 0; e < 8; e += Vec<O>::N) Vec<O>::store(o + j + e, v + e);
      }
      done = n / 8 * 8;
    }
    for (int j = done + threadIdx.x; j < n; j += 256) o[j] = (O)((float)g[j] * c);
  }
}

static int grid_of(const GradTable& t) { return t.pieces < kGradSums ? t.pieces : kGradSums; }

// Walks the list in tables of kGradTable tensors: body(table, workgroups, sums before it).
template <typename F>
static hipError_t tables(int n, const void* const* src, void* const* dst, const int64_t* counts, F body) {
  int sums = 0;
  for (int i = 0; i < n;) {
    GradTable t{};
    for (; i < n && t.n < kGradTable; i++) {
      if (counts[i] == 0) continue;
      const int64_t pieces = (counts[i] + kPiece - 1) / kPiece;
      if (t.pieces + pieces > (1 << 30)) break;
      t.src[t.n] = src[i]; t.dst[t.n] = dst ? dst[i] : nullptr; t.count[t.n] = counts[i]; t.first[t.n] = t.pieces;
      t.pieces += (int)pieces;
      t.n++;
    }
    if (t.n == 0) continue;
    if (hipError_t e = body(t, grid_of(t), sums); e != hipSuccess) return e;
    sums += grid_of(t);
  }
  return hipSuccess;
}

hipError_t grad_sumsq(int dtype, int n, const void* const* grads, const int64_t* counts, double* sums, int* n_sums, hipStream_t s) {
  *n_sums = 0;
  return tables(n, grads, nullptr, counts, [&](const GradTable& t, int grid, int before) {
    if (dtype) hipLaunchKernelGGL((grad_sumsq_kernel<bf16_t>), dim3((unsigned)grid), dim3(256), 0, s, t, sums + before);
    else hipLaunchKernelGGL((grad_sumsq_kernel<float>), dim3((unsigned)grid), dim3(256), 0, s, t, sums + before);
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
  const hipError_t e = tables(n, grads, outs, counts, [&](const GradTable& t, int grid, int) {
    float* const out = first ? norm : nullptr;
    first = false;
    const dim3 g((unsigned)grid), b(256);
    if (dtype && out_dtype) hipLaunchKernelGGL((grad_clip_kernel<bf16_t, bf16_t>), g, b, 0, s, t, sums, n_sums, max_norm, out);
    else if (dtype) hipLaunchKernelGGL((grad_clip_kernel<bf16_t, float>), g, b, 0, s, t, sums, n_sums, max_norm, out);
    else if (out_dtype) hipLaunchKernelGGL((grad_clip_kernel<float, bf16_t>), g, b, 0, s, t, sums, n_sums, max_norm, out);
    else hipLaunchKernelGGL((grad_clip_kernel<float, float>), g, b, 0, s, t, sums, n_sums, max_norm, out);
    return hipGetLastError();
  });
  if (e != hipSuccess || !first) return e;
  GradTable none{};                                             // nothing to clip: the norm alone
  hipLaunchKernelGGL((grad_clip_kernel<float, float>), dim3(1), dim3(256), 0, s, none, sums, n_sums, max_norm, norm);
  return hipGetLastError();
}

}  // namespace tbp
