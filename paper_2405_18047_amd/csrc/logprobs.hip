// Log probabilities of given tokens over rows of logits, with the entropy of every row and its most likely tokens, and the
// derivative of the logits.
//   m = max x, s = sum e^(x - m), t = sum (x - m) e^(x - m):  lse = m + log s,  logp = x_target - lse,  H = log s - t / s,
//   dx = dlogp (1[target] - p) - dH p (log p + H).
// All of them are read (and written) once at the memory's rate in the end; statistics are fp32.
#include "kernels.h"
#include "rows.h"

namespace tbp {

struct Stats { float m, s, t; };
__device__ __forceinline__ Stats join(Stats a, Stats b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return Stats{m, a.s + b.s, a.t + b.t};       // (nothing but -inf so far: zeros, or NaN that is passed on)
  const float da = a.m - m, db = b.m - m, fa = __expf(da), fb = __expf(db);
  return Stats{m, a.s * fa + b.s * fb, (a.m == -INFINITY ? 0.f : (a.t + da * a.s) * fa) + (b.m == -INFINITY ? 0.f : (b.t + db * b.s) * fb)};
}
__device__ __forceinline__ void add(Stats& a, float x) {
  if (x == -INFINITY) return;
  if (x > a.m) {
    const float d = a.m - x, f = __expf(d);
    a.t = a.m == -INFINITY ? a.t : (a.t + d * a.s) * f;
    a.s = a.s * f;
    a.m = x;
  }
  const float d = x - a.m, e = __expf(d);
  a.s += e;
  a.t += d * e;
}

// a is ranked before b: larger value, or the same and a lower index
__device__ __forceinline__ bool before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

template <typename T>
__global__ __launch_bounds__(256) void logprobs_kernel(LogprobParams p) {
  __shared__ Stats red[4];
  __shared__ float bv[4];
  __shared__ int bi[4];
  const long row = blockIdx.x;
  const T* const x = (const T*)p.logits + row * p.ld;
  Stats a{-INFINITY, 0.f, 0.f};
  for (int i = threadIdx.x; i < p.vocab; i += 256) add(a, (float)x[i]);
  for (int d = 1; d < 64; d <<= 1) a = join(a, Stats{__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.t, d)});
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = a;
  __syncthreads();
  a = join(join(red[0], red[1]), join(red[2], red[3]));
  const float ls = logf(a.s), lse = a.m == -INFINITY ? (a.s == a.s ? -INFINITY : a.s) : a.m + ls;
  if (threadIdx.x == 0) {
    const int t = p.targets ? p.targets[row] : -1;
    if (p.logp) p.logp[row] = t >= 0 && t < p.vocab ? (lse == -INFINITY ? -INFINITY : (float)x[t] - lse) : 0.f;
    if (p.entropy) p.entropy[row] = lse == -INFINITY ? 0.f : ls - a.t / a.s;
    if (p.lse) p.lse[row] = lse;
  }
  float pv = INFINITY;
  int pi = -1;
  for (int k = 0; k < p.top; k++) {
    float v = -INFINITY;
    int best = 0x7fffffff;
    for (int i = threadIdx.x; i < p.vocab; i += 256) {
      const float c = (float)x[i];
      if ((c < pv || (c == pv && i > pi)) && (best == 0x7fffffff || before(c, i, v, best))) { v = c; best = i; }
    }
    for (int d = 1; d < 64; d <<= 1) {
      const float ov = __shfl_xor(v, d);
      const int oi = __shfl_xor(best, d);
      if (before(ov, oi, v, best)) { v = ov; best = oi; }
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { bv[threadIdx.x >> 6] = v; bi[threadIdx.x >> 6] = best; }
    __syncthreads();
    v = bv[0]; best = bi[0];
    for (int w = 1; w < 4; w++)
      if (before(bv[w], bi[w], v, best)) { v = bv[w]; best = bi[w]; }
    if (threadIdx.x == 0) {
      const bool ok = lse == lse && best < p.vocab;
      p.top_logp[row * p.top + k] = !ok ? __builtin_nanf("") : lse == -INFINITY ? -INFINITY : v - lse;
      p.top_ids[row * p.top + k] = ok ? best : -1;
    }
    pv = v; pi = best;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void logprobs_p1_kernel(LogprobParams p) {
  const long row = blockIdx.x;
  const int i = (int)blockIdx.y * 256 + threadIdx.x;
  if (i >= p.vocab) return;
  const float lse = p.lse[row], x = (float)((const T*)p.logits)[row * p.ld + i];
  const int t = p.targets[row];
  const float dl = t >= 0 && t < p.vocab ? p.d_logp[row] : 0.f, dh = p.d_entropy ? p.d_entropy[row] : 0.f;
  const float lp = x - lse, pr = __expf(lp);
  float d = pr > 0.f ? -pr * (dl + dh * (lp + p.entropy[row])) : 0.f;
  if (pr != pr) d = pr;
  if (i == t) d += dl;
  ((T*)p.d_logits)[row * p.ld_d + i] = (T)(lse == -INFINITY ? 0.f : d);
}

hipError_t logprobs(int dtype, const LogprobParams& p, hipStream_t s) {
  if (dtype) hipLaunchKernelGGL((logprobs_kernel<bf16_t>), dim3((unsigned)p.rows), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((logprobs_kernel<float>), dim3((unsigned)p.rows), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t logprobs_p1(int dtype, const LogprobParams& p, hipStream_t s) {
  const dim3 grid((unsigned)p.rows, (unsigned)((p.vocab + 255) / 256));
  if (dtype) hipLaunchKernelGGL((logprobs_p1_kernel<bf16_t>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((logprobs_p1_kernel<float>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t logprobs_step(int dtype, const LogprobParams& p, hipStream_t s) {
  if (hipError_t e = logprobs(dtype, p, s); e != hipSuccess) return e;
  return logprobs_p1(dtype, p, s);
}

}  // namespace tbp
