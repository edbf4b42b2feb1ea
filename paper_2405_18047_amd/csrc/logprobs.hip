// Log probabilities of given tokens over rows of logits, with the entropy of every row and its most likely tokens, and the
// derivative of the logits.  With the maximum m of a row and d = (x - m) log2 e,
//   s = sum 2^d, t = sum d 2^d:   lse = m + ln s,  logp = (x_target - m) - ln s,  H = (log2 s - t / s) ln 2,
//   dx = dlogp (1[target] - p) - dH p (log p + H),  p = 2^(d - log2 s).
// The difference comes first: it is as exact as the logits for those that count, and a row of nothing but the type's lowest value (a mask
// that leaves nothing) is the uniform distribution that it says.
//
// A workgroup owns a row and holds it in registers (16 or 4 pieces of 16 bytes per thread) from the statistics to the ranking or to the
// derivative: a row is read once.  Rows longer than that are walked in blocks and read a second time for the derivative (for the ranking
// only by the few threads that hold a candidate).
#include "kernels.h"
#include "rows.h"

#include <type_traits>

namespace tbp {

// 2^d is zero below this: what it is multiplied with only has to be finite there (a logit of -infinity).  A NaN stays one by 2^d.
constexpr float kFar = -300.f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 16 bytes at any address that an element may have (rows of odd length): one load or store all the same.
typedef u32x4 Any4 __attribute__((aligned(4)));
typedef u32x4 Any2 __attribute__((aligned(2)));
template <typename T> struct Logits {
  static constexpr int N = 16 / (int)sizeof(T);
  typedef typename std::conditional<sizeof(T) == 4, Any4, Any2>::type Any;
  static __device__ __forceinline__ u32x4 load(const T* p) { return *reinterpret_cast<const Any*>(p); }
  // (nontemporal: [4096, 32000] bf16 with its derivative 109.6 -> 88.6 us; loads of that kind, 109.6 -> 97.0)
  static __device__ __forceinline__ void store(T* p, const float* v) {
    if constexpr (sizeof(T) == 4) {
      const u32x4 o{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
      __builtin_nontemporal_store(o, reinterpret_cast<Any*>(p));
    } else {
      typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
      bf16x8 o;
#pragma unroll
      for (int i = 0; i < 8; i++) o[i] = (bf16_t)v[i];
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, o), reinterpret_cast<Any*>(p));
    }
  }
  static __device__ __forceinline__ float get(const u32x4& r, int i) {      // i is a constant after unrolling
    if constexpr (sizeof(T) == 4) return __uint_as_float(r[i]);
    else return (i & 1) ? __uint_as_float(r[i >> 1] & 0xffff0000u) : __uint_as_float(r[i >> 1] << 16);
  }
  static constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;      // -infinity
};

// Statistics of a part of a row; m = -infinity: nothing above it so far (s, t: zeros, or NaN that is passed on).
struct Stats { float m, s, t; };
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b) {
  const float m = fmaxf(a.m, b.m);
  // (of the two one is m; the other's difference may be infinite: then its factor is zero and only has to stay clear of 0 * infinity)
  const float da = a.m == -INFINITY ? 0.f : fmaxf((a.m - m) * kLog2e, kFar), db = b.m == -INFINITY ? 0.f : fmaxf((b.m - m) * kLog2e, kFar);
  const float fa = a.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(da), fb = b.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(db);
  return Stats{m, a.s * fa + b.s * fb, (a.t + da * a.s) * fa + (b.t + db * b.s) * fb};
}

// a is ranked before b: larger value, or the same and a lower index
__device__ __forceinline__ bool before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

// What the threads of a row share: for the statistics, and for the ranking.
template <int NT> struct RowShared { Stats red[NT / 64]; };
template <int NT> struct RankShared {
  static constexpr int kCandidates = NT == 64 ? 256 : 1024;
  float lane_max[NT / 64][64];
  float bar;
  int n;
  uint64_t key[kCandidates];
  float bv[NT / 64];
  int bi[NT / 64];
};

// Value and index as one number: larger for what is ranked before.  (The value's bits as an unsigned number in the order of the values; no
// NaN comes here, and -0 counts as 0.)
__device__ __forceinline__ uint64_t rank_key(float v, int i) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~i;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

// One row's pieces: piece c of the thread's block b is at element N (NT (CH b + c) + thread).
template <typename T, int NT, int CH>
struct Row {
  using L = Logits<T>;
  static constexpr int N = L::N;
  u32x4 x[CH];
  // The pieces as they are, but unknown to the compiler: what one pass has unpacked from them is not kept for the next (twice the registers).
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (int c = 0; c < CH; c++) asm volatile("" : "+v"(x[c]));
  }
  __device__ __forceinline__ float piece_max(int c) const {
    float m = L::get(x[c], 0);
#pragma unroll
    for (int e = 1; e < N; e++) m = fmaxf(m, L::get(x[c], e));
    return m;
  }
  static __device__ __forceinline__ int at(int blk, int c) { return N * (NT * (CH * blk + c) + (int)threadIdx.x); }
  __device__ __forceinline__ void load(const T* row, int vocab, int blk) {
#pragma unroll
    for (int c = 0; c < CH; c++) {
      const int i = at(blk, c);
      if (i + N <= vocab) x[c] = L::load(row + i);
      else x[c] = u32x4{L::kNone, L::kNone, L::kNone, L::kNone};
    }
    // the row's end, if it lies inside a piece
    const int tail = vocab / N * N;
    if (tail < vocab && tail / N % NT == (int)threadIdx.x && tail / N / NT / CH == blk) {
#pragma unroll
      for (int c = 0; c < CH; c++) {
        if (at(blk, c) != tail) continue;
#pragma unroll
        for (int e = 0; e < N - 1; e++) {
          if (tail + e >= vocab) continue;
          if constexpr (sizeof(T) == 4) x[c][e] = reinterpret_cast<const uint32_t*>(row)[tail + e];
          else {
            const uint32_t v = reinterpret_cast<const uint16_t*>(row)[tail + e];
            x[c][e >> 1] = (e & 1) ? (x[c][e >> 1] & 0xffffu) | v << 16 : (x[c][e >> 1] & 0xffff0000u) | v;
          }
        }
      }
    }
  }
};

// Ranking.  The row's maxima over 64 (or 128) classes of threads are so many of its logits, so the top-th largest of them is a lower bound of
// the top-th largest logit, and hardly more logits than `top` reach it: as many as draws from 64 boxes take until `top` have been
// met, 24 for 20 and 44 for 32 (of 128 boxes 89 for 64).  Those are collected and ranked among each other.  Rows with more of them than there is
// room for (a great many ties) are ranked one place at a time over the whole row.
template <typename T, int NT, int CH>
__device__ __forceinline__ void rank_top(const LogprobParams& p, long row, const T* x, Row<T, NT, CH>& data, const float (&piece_max)[CH], int nblk, float my_max, float lse, float m, float ln_s,
                                         RankShared<NT>& sh) {
  using R = Row<T, NT, CH>;
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  float* const out_v = p.top_logp + row * p.top;
  int* const out_i = p.top_ids + row * p.top;
  if (!(lse == lse)) {                               // NaN or +infinity in the row
    if (tid < p.top) { out_v[tid] = __builtin_nanf(""); out_i[tid] = -1; }
    return;
  }
  // the bar: the waves rank the classes among them, 64 / NW (128 / NW) each, and whoever finds the one in place top - 1 says so
  if (tid == 0) sh.n = 0;
  const int classes = NW > 1 && p.top > 32 ? 128 : 64;
  if constexpr (NW > 1) {
    sh.lane_max[wave][lane] = my_max;
    __syncthreads();
  }
  float cls[2] = {my_max, -INFINITY};
  if constexpr (NW > 1) {
    cls[0] = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; w++) cls[w & 1] = fmaxf(cls[w & 1], sh.lane_max[w][lane]);
    if (classes == 64) cls[0] = fmaxf(cls[0], cls[1]);
  }
  if constexpr (NW == 1) {                           // one wave: every lane finds its own class's rank
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < 64; j++)
      rank += before(__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, my_max), j)), j, my_max, lane) ? 1 : 0;
    if (rank == p.top - 1) sh.bar = my_max;
  }
  for (int j = wave; NW > 1 && j < classes; j += NW) {
    const float mine = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, j < 64 ? cls[0] : cls[1]), j & 63));
    int rank = __popcll(__ballot(before(cls[0], lane, mine, j)));
    if (classes == 128) rank += __popcll(__ballot(before(cls[1], 64 + lane, mine, j)));
    if (rank == p.top - 1) sh.bar = mine;
  }
  __syncthreads();
  const float bar = sh.bar;
  // (bar -infinity: fewer than `top` classes hold a finite logit; the finite ones are collected and the rest of the places filled below)
  if (my_max >= bar && my_max > -INFINITY) {
    for (int b = 0; b < nblk; b++) {
      if (nblk > 1) data.load(x, p.vocab, b);
      data.forget();
#pragma unroll
      for (int c = 0; c < CH; c++) {
        if ((nblk > 1 ? data.piece_max(c) : piece_max[c]) < bar) continue;
#pragma unroll
        for (int e = 0; e < R::N; e++) {
          const float v = Logits<T>::get(data.x[c], e);
          if (v >= bar && v > -INFINITY) {
            const int at = atomicAdd(&sh.n, 1);
            if (at < sh.kCandidates) sh.key[at] = rank_key(v, R::at(b, c) + e);
          }
        }
      }
    }
  }
  __syncthreads();
  const int n = __builtin_amdgcn_readfirstlane(sh.n);
  if (n <= sh.kCandidates) {
    for (int i = wave; i < n; i += NW) {             // a wave counts what is ranked before candidate i
      const uint64_t mine = sh.key[i];
      int rank = 0;
      for (int j0 = 0; j0 < n; j0 += 64) rank += __popcll(__ballot(j0 + lane < n && sh.key[j0 + lane] > mine));
      if (lane == 0 && rank < p.top) { out_v[rank] = (key_value(mine) - m) - ln_s; out_i[rank] = (int)~(uint32_t)mine; }
    }
    // fewer finite logits than places: the others in order of their index, which are among the first n + top
    if (n < p.top && wave == 0) {
      int place = n;
      for (int i0 = 0; place < p.top; i0 += 64) {
        const bool none = i0 + lane < p.vocab && (float)x[i0 + lane] == -INFINITY;
        const uint64_t who = __ballot(none);
        const int at = place + __popcll(who & ((1ull << lane) - 1));
        if (none && at < p.top) { out_v[at] = -INFINITY; out_i[at] = i0 + lane; }
        place += __popcll(who);
      }
    }
    return;
  }
  float pv = INFINITY;
  int pi = -1;
  for (int k = 0; k < p.top; k++) {
    float v = -INFINITY;
    int best = 0x7fffffff;
    for (int i = tid; i < p.vocab; i += NT) {
      const float c = (float)x[i];
      if ((c < pv || (c == pv && i > pi)) && (best == 0x7fffffff || before(c, i, v, best))) { v = c; best = i; }
    }
    for (int d = 1; d < 64; d <<= 1) {
      const float ov = __shfl_xor(v, d);
      const int oi = __shfl_xor(best, d);
      if (before(ov, oi, v, best)) { v = ov; best = oi; }
    }
    __syncthreads();
    if ((tid & 63) == 0) { sh.bv[tid >> 6] = v; sh.bi[tid >> 6] = best; }
    __syncthreads();
    v = sh.bv[0]; best = sh.bi[0];
    for (int w = 1; w < NT / 64; w++)
      if (before(sh.bv[w], sh.bi[w], v, best)) { v = sh.bv[w]; best = sh.bi[w]; }
    if (tid == 0) { out_v[k] = lse == -INFINITY ? -INFINITY : (v - m) - ln_s; out_i[k] = best; }
    pv = v; pi = best;
  }
}

// The derivative of one piece of a row.
struct RowWeights { float m, ls, dl, inner, dh2; int target; };     // p = 2^((x - m) log2 e - ls); inner = dl + dH H, dh2 = dH ln 2
__device__ __forceinline__ RowWeights row_weights(const LogprobParams& p, long row, float m, float ls, float entropy) {
  const int t = p.targets[row];
  const bool given = t >= 0 && t < p.vocab, none = m == -INFINITY;
  const float dl = given && !none ? p.d_logp[row] : 0.f, dh = p.d_entropy && !none ? p.d_entropy[row] : 0.f;
  return RowWeights{none ? 0.f : m, none ? 0.f : ls, dl, dl + dh * entropy, dh * kLn2, given ? t : -1};
}
template <typename T>
__device__ __forceinline__ void derive(const u32x4& x, int i, const RowWeights& w, float* v) {
  using L = Logits<T>;
#pragma unroll
  for (int e = 0; e < L::N; e++) {
    const float d = __builtin_fmaf(L::get(x, e) - w.m, kLog2e, -w.ls);
    v[e] = -__builtin_amdgcn_exp2f(d) * __builtin_fmaf(w.dh2, fmaxf(d, kFar), w.inner);
  }
  if ((unsigned)(w.target - i) < (unsigned)L::N) {
#pragma unroll
    for (int e = 0; e < L::N; e++) v[e] += w.target - i == e ? w.dl : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_piece(T* row, int i, int vocab, const float* v) {
  using L = Logits<T>;
  if (i + L::N <= vocab) L::store(row + i, v);
  else
#pragma unroll
    for (int e = 0; e < L::N - 1; e++)
      if (i + e < vocab) row[i + e] = (T)v[e];
}

// Bound where rows are many by memory and as nearly by the vector instructions, issued in 95 % of the cycles: statistics and derivative of [4096, 32000] bf16
// (524 MB read and written, a row on 256 threads of 16 pieces) 97 us, 5.4 TB/s; by the chain of a row's passes where they are few: 20 candidates of each of 7 rows of 50257 fp32 12 us, 1.4 MB.
template <typename T, int NT, int CH, bool STEP>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(4))) void logprobs_kernel(LogprobParams p) {
  using R = Row<T, NT, CH>;
  __shared__ RowShared<NT> sh;
  const int tid = threadIdx.x;
  const long row = blockIdx.x;
  const T* const x = (const T*)p.logits + row * p.ld;
  const int nblk = (p.vocab + NT * CH * R::N - 1) / (NT * CH * R::N);
  R data;
  Stats a{-INFINITY, 0.f, 0.f};
  float my_max = -INFINITY, piece_max[CH];            // (of the last block)
  for (int b = 0; b < nblk; b++) {
    data.load(x, p.vocab, b);
    float mx = my_max;
#pragma unroll
    for (int c = 0; c < CH; c++) {
      piece_max[c] = data.piece_max(c);
      mx = fmaxf(mx, piece_max[c]);
    }
    if (mx > my_max) {                               // the reference point moves to the maximum
      const float d = a.m == -INFINITY ? 0.f : fmaxf((a.m - mx) * kLog2e, kFar), f = __builtin_amdgcn_exp2f(d);
      a.t = (a.t + d * a.s) * f;
      a.s *= f;
      a.m = mx;
      my_max = mx;
    }
    data.forget();
    const float ref = a.m == -INFINITY ? 0.f : a.m;
    float s[2] = {0.f, 0.f}, t = 0.f;
#pragma unroll
    for (int c = 0; c < CH; c++)
#pragma unroll
      for (int e = 0; e < R::N; e++) {
        const float d = (Logits<T>::get(data.x[c], e) - ref) * kLog2e, v = __builtin_amdgcn_exp2f(d);
        s[e & 1] += v;
        t = __builtin_fmaf(v, fmaxf(d, kFar), t);
      }
    a.s += s[0] + s[1];
    a.t += t;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) a = join(a, Stats{__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.t, d)});
  if ((tid & 63) == 0) sh.red[tid >> 6] = a;
  __syncthreads();
  a = sh.red[tid & (NT / 64 - 1)];
#pragma unroll
  for (int d = 1; d < NT / 64; d <<= 1) a = join(a, Stats{__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.t, d)});
  // (lane 0's sums for all: lanes may differ in the last bit)
  auto first = [](float v) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v))); };
  a = Stats{first(a.m), first(a.s), first(a.t)};
  const bool none = a.m == -INFINITY && a.s == a.s;                 // nothing but -infinity
  const float ls = __builtin_amdgcn_logf(a.s);
  const float lse = none ? -INFINITY : a.m == -INFINITY ? a.s : a.m + ls * kLn2, entropy = none ? 0.f : (ls - a.t / a.s) * kLn2;
  if (tid == 0) {
    const int t = p.targets[row];
    p.logp[row] = t >= 0 && t < p.vocab ? (none ? -INFINITY : ((float)x[t] - a.m) - ls * kLn2) : 0.f;
    p.entropy[row] = entropy;
    p.lse[row] = lse;
  }
  if constexpr (STEP) {
    __syncthreads();                                                // (in place: the target's logit has been read)
    const RowWeights w = row_weights(p, row, lse == lse ? a.m : lse, ls, entropy);
    T* const o = (T*)p.d_logits + row * p.ld_d;
    for (int b = 0; b < nblk; b++) {
      if (nblk > 1) data.load(x, p.vocab, b);
      data.forget();
#pragma unroll
      for (int c = 0; c < CH; c++) {
        const int i = R::at(b, c);
        if (i >= p.vocab) break;
        float v[R::N];
        derive<T>(data.x[c], i, w, v);
        store_piece<T>(o, i, p.vocab, v);
      }
    }
  } else {
    __shared__ RankShared<NT> rank;
    if (p.top) rank_top<T, NT, CH>(p, row, x, data, piece_max, nblk, my_max, lse, a.m, ls * kLn2, rank);
  }
}

// The derivative by itself: a workgroup takes 4 pieces per thread of one row, for rows and parts of rows are all alike here.  Bound by memory:
// [1023, 131072] bf16, 536 MB read and written, 100 us, 5.4 TB/s.
// p comes from x - lse, as exact as lse is: below kCoarse half of its last place is 2^-15 at most.  A row beyond (nothing but the type's lowest
// value, say, where lse does not show ln s at all) is one workgroup's alone, which sums it up again first; alone, for d_logits may be the logits.
constexpr float kCoarse = 1024.f;
template <typename T>
__global__ __launch_bounds__(256) void logprobs_p1_kernel(LogprobParams p) {
  using R = Row<T, 256, 4>;
  const long row = blockIdx.x;
  const T* const x = (const T*)p.logits + row * p.ld;
  T* const o = (T*)p.d_logits + row * p.ld_d;
  R data;
  auto derivative = [&](int blk, const RowWeights& w) {
#pragma unroll
    for (int c = 0; c < 4; c++) {
      const int i = R::at(blk, c);
      if (i >= p.vocab) break;
      float v[R::N];
      derive<T>(data.x[c], i, w, v);
      store_piece<T>(o, i, p.vocab, v);
    }
  };
  data.load(x, p.vocab, blockIdx.y);
  const float lse = p.lse[row], entropy = p.entropy[row];
  if (!(__builtin_fabsf(lse) >= kCoarse && __builtin_fabsf(lse) < INFINITY)) {
    derivative(blockIdx.y, row_weights(p, row, lse, 0.f, entropy));
    return;
  }
  if (blockIdx.y) return;
  __shared__ float red[2][4];
  const int tid = threadIdx.x;
  float m = -INFINITY, s = 0.f;
  for (int i = tid; i < p.vocab; i += 256) m = fmaxf(m, (float)x[i]);
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  if ((tid & 63) == 0) red[0][tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  for (int i = tid; i < p.vocab; i += 256) s += __builtin_amdgcn_exp2f(((float)x[i] - m) * kLog2e);
  for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
  if ((tid & 63) == 0) red[1][tid >> 6] = s;
  __syncthreads();                                                  // (in place: the whole row has been read)
  s = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  const RowWeights w = row_weights(p, row, m, __builtin_amdgcn_logf(s), entropy);
  for (int b = 0; b < (int)gridDim.y; b++) {
    data.load(x, p.vocab, b);
    derivative(b, w);
  }
}

// The rows from r0 on (a launch takes at most kLaunchRows of them: its threads are counted in 32 bits).  r0 runs past the largest row count.
constexpr int kLaunchRows = 1 << 21;
static LogprobParams rows_from(LogprobParams p, long r0, int element) {
  p.rows = p.rows - r0 < kLaunchRows ? (int)(p.rows - r0) : kLaunchRows;
  p.logits = (const char*)p.logits + r0 * p.ld * element;
  p.targets += r0; p.entropy += r0; p.lse += r0;
  if (p.logp) p.logp += r0;
  if (p.top) { p.top_logp += r0 * p.top; p.top_ids += r0 * p.top; }
  if (p.d_logp) p.d_logp += r0;
  if (p.d_entropy) p.d_entropy += r0;
  if (p.d_logits) p.d_logits = (char*)p.d_logits + r0 * p.ld_d * element;
  return p;
}

template <typename T, int NT, int CH, bool STEP>
static hipError_t launch(const LogprobParams& p, hipStream_t s) {
  for (long r0 = 0; r0 < p.rows; r0 += kLaunchRows) {
    const LogprobParams q = rows_from(p, r0, sizeof(T));
    hipLaunchKernelGGL((logprobs_kernel<T, NT, CH, STEP>), dim3((unsigned)q.rows), dim3(NT), 0, s, q);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Threads and pieces per thread of a row (256 x 4: 1024 N logits at a time, longer rows in blocks), chosen by length, by whether there are more rows than
// compute units, and by what follows the statistics: the derivative reads a row that is not held a second time, the ranking costs a narrow workgroup
// more than a wide one, and statistics alone gain nothing by holding the row, while pieces behind its end cost as much as others.  us, bf16 (N = 8), rows x
// logits / N, the chosen form and the other that is nearest; fp32 and rows of odd length (unaligned) put the same ones ahead:
//   statistics   7 x 256 64x4 3.9, 256x4 4.2; 4096 x 256 7.6, 17.0; 7 x 1024 256x4 4.2, 64x16 5.8; 4096 x 512 64x16 14.7, 256x4 17.2, x 1024 18.3, 18.2;
//                7 x 2000 256x4 5.4, 1024x4 6.3; 300 x 2000 7.1, 256x16 9.4; 7 x 4096 1024x4 6.3, 256x4 7.1; 300 x 4096 256x16 10.6, 256x4 10.3, 4096 x 4096
//                54.0, 56.5; 7 x 6000 512x16 8.1, 1024x16 12.1; 300 x 6000 256x4 12.9, 512x16 15.3; 7 x 16600 1024x4 15.9, 1024x16 21.8; 300 x 16600 32.6, 256x16 31.4
//   20 ranked    7 x 256 256x4 8.4, 64x4 13.3; 4096 x 256 64x4 22.2, 256x4 28.2; 300 x 1024 256x4 11.1, 64x16 20.7; 7 x 2000 1024x4 9.6, 256x4 12.0; 300 x 2000
//                256x4 14.7, 256x16 16.5; 7 x 4096 1024x4 9.9, 256x16 13.4; 300 x 4096 256x16 18.0, 1024x4 15.8, 4096 x 4096 73.6, 90.5; 300 x 6000 512x16 22.1,
//                256x16 27.3; 7 x 16032 1024x16 17.8, 1024x4 21.0; 300 x 16032 1024x4 37.4, 256x16 43.3; 7 x 16600 24.4, 1024x16 32.8
//   derivative   300 x 256 64x4 5.3, 256x4 5.7; 300 x 1024 256x4 7.2, 64x16 10.3; 4096 x 1024 64x16 27.6, 256x4 30.0; 7 x 4096 1024x4 9.0, 256x16 10.1; 4096 x 4096
//                256x16 106.6, 1024x4 116.5; 7 x 6000 512x16 12.1, 1024x4 12.9, 4096 x 6000 170, 184; 300 x 16032 1024x16 50.0, 1024x4 55.2; 300 x 16600 1024x4 60.6,
//                256x16 63.2, 1024x16 77.3
template <typename T, bool STEP>
static hipError_t launch_t(const LogprobParams& p, hipStream_t s) {
  constexpr int N = Logits<T>::N;
  const bool many = p.rows > 256, crowd = p.rows > 2048, top = p.top > 0;
  if (p.vocab <= 256 * N && (!top || (crowd && p.top <= 32))) return launch<T, 64, 4, STEP>(p, s);
  if (p.vocab <= 1024 * N) return crowd && !top ? launch<T, 64, 16, STEP>(p, s) : launch<T, 256, 4, STEP>(p, s);
  if constexpr (STEP) {
    if (p.vocab <= 4096 * N) return many ? launch<T, 256, 16, STEP>(p, s) : launch<T, 1024, 4, STEP>(p, s);
    if (p.vocab <= 8192 * N) return launch<T, 512, 16, STEP>(p, s);
    return p.vocab <= 16384 * N ? launch<T, 1024, 16, STEP>(p, s) : launch<T, 1024, 4, STEP>(p, s);
  } else {
    if (p.vocab <= 2048 * N) return many || !top ? launch<T, 256, 4, STEP>(p, s) : launch<T, 1024, 4, STEP>(p, s);
    if (p.vocab <= 4096 * N) return many ? launch<T, 256, 16, STEP>(p, s) : launch<T, 1024, 4, STEP>(p, s);
    if (p.vocab <= 8192 * N) return many && !top ? launch<T, 256, 4, STEP>(p, s) : launch<T, 512, 16, STEP>(p, s);
    return p.vocab <= 16384 * N && !many && top ? launch<T, 1024, 16, STEP>(p, s) : launch<T, 1024, 4, STEP>(p, s);
  }
}

hipError_t logprobs(int dtype, const LogprobParams& p, hipStream_t s) { return dtype ? launch_t<bf16_t, false>(p, s) : launch_t<float, false>(p, s); }
hipError_t logprobs_step(int dtype, const LogprobParams& p, hipStream_t s) { return dtype ? launch_t<bf16_t, true>(p, s) : launch_t<float, true>(p, s); }

hipError_t logprobs_p1(int dtype, const LogprobParams& p, hipStream_t s) {
  const int per = 256 * 4 * (dtype ? 8 : 4);
  for (long r0 = 0; r0 < p.rows; r0 += kLaunchRows) {
    const LogprobParams q = rows_from(p, r0, dtype ? 2 : 4);
    const dim3 grid((unsigned)q.rows, (unsigned)((p.vocab + per - 1) / per));
    if (dtype) hipLaunchKernelGGL((logprobs_p1_kernel<bf16_t>), grid, dim3(256), 0, s, q);
    else hipLaunchKernelGGL((logprobs_p1_kernel<float>), grid, dim3(256), 0, s, q);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace tbp
