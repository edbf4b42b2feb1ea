// A stash in 8 bits for gfx950: a linear layer's inputs and output derivatives are kept from backward-p1 to backward-p2 as 8-bit integers,
// and the weight gradient dW = X^T dY is formed from them on the integer matrix instructions.
//
// Of every kStash8Block tokens of a column (counted from a slot's first token) the values are q 2^e with q = -127 .. 127 and e the smallest exponent,
// -126 at least, with which the largest of them is in that range (121 at most: beyond, q ends at 127); q is the nearest integer, halves to even.  Powers of two, so that scaling is exact and
// the one rounding is q's: at most half of 2^e.  For e above -126 the largest value is above 127 2^(e - 1), so that 2^e is below 1/63.5 of it; at -126 the half step is 2^-127,
// whatever the values; at 121 a value above 127 2^121 is off by what it is above that.
// A block that holds an infinity or a NaN has no such scale: its scale is NaN, and with it all that it stands for.
//
// Layout: the matrix instructions want, per column, consecutive tokens.  A unit of 32 columns x 64 tokens is 2 KiB: two halves of 32 tokens, in each the
// 16 bytes of lane l = tokens 16 (l / 32) .. of column l % 32, as the instruction's operand lies in its registers.  Units lie column block after column
// block, then 64 tokens after 64 tokens, then slot after slot (a slot's tokens are padded with zeros to a multiple of 64), so that the slots of a step are
// one contraction length.  Behind them the scales, fp32: [slot][block of tokens][column].
#include "kernels.h"
#include "rows.h"

#include <type_traits>

namespace tbp {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kUnit = 2048;                      // bytes of a unit
constexpr int kStepsPerBlock = kStash8Block / 64;
constexpr int kTopExponent = 121;                // of a scale: 127 2^121 is the largest multiple that fp32 has

// ------------------------------------------------------------------------------------------ into the stash, and out of it
// One workgroup = 64 columns of one block of tokens, 8 threads side by side with 8 columns each (128 bytes of a row, bf16) and 64 of them below each other
// with 16 tokens each, which stay in registers as they were loaded between the two looks at them: the largest magnitude of every column, then the rounding.
// Bound by memory: 4096 x 11008 of bf16, 135 MB read and written, 22.4 us, 6.0 TB/s (of new inputs, out of no cache, 27 to 32); few tokens by a workgroup's chain of a load,
// two barriers and a store: 129 x 256 5 us.
// Magnitudes are compared as bit patterns, in which NaN is above infinity (bf16: two to an instruction).
template <typename T> struct Rows8;              // 8 columns of a row as they lie in memory
template <> struct Rows8<bf16_t> {
  typedef u32x4 Raw __attribute__((aligned(2)));      // (the memory instructions take any alignment)
  u32x4 q;
  __device__ __forceinline__ void load(const bf16_t* p) { q = *reinterpret_cast<const Raw*>(p); }
  // the first n columns without, zeros behind them
  __device__ __forceinline__ void drop(int n) {
    if (n & 4) q = u32x4{q[2], q[3], 0, 0};
    if (n & 2) q = u32x4{q[1], q[2], q[3], 0};
    if (n & 1) q = u32x4{__builtin_amdgcn_alignbit(q[1], q[0], 16), __builtin_amdgcn_alignbit(q[2], q[1], 16), __builtin_amdgcn_alignbit(q[3], q[2], 16), q[3] >> 16};
  }
  __device__ __forceinline__ void set(int c, bf16_t v) {
    const unsigned b = (unsigned)__builtin_bit_cast(unsigned short, v);
    q[c / 2] = c % 2 ? (q[c / 2] & 0xffffu) | (b << 16) : (q[c / 2] & 0xffff0000u) | b;
  }
  __device__ __forceinline__ void clear() { q = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ float get(int c) const { return __uint_as_float(c % 2 ? q[c / 2] & 0xffff0000u : q[c / 2] << 16); }
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  struct Top {
    u32x4 m = {0, 0, 0, 0};
    static __device__ __forceinline__ unsigned more(unsigned a, unsigned b) {
      return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    }
    __device__ __forceinline__ void add(const Rows8& r) {
#pragma unroll
      for (int i = 0; i < 4; i++) m[i] = more(m[i], r.q[i] & 0x7fff7fffu);
    }
    __device__ __forceinline__ void across(int d) {
#pragma unroll
      for (int i = 0; i < 4; i++) m[i] = more(m[i], (unsigned)__shfl_xor((int)m[i], d));
    }
    __device__ __forceinline__ unsigned get(int c) const { return c % 2 ? m[c / 2] & 0xffff0000u : m[c / 2] << 16; }
  };
};
template <> struct Rows8<float> {
  typedef u32x4 Raw __attribute__((aligned(4)));
  u32x4 q[2];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < 2; i++) q[i] = *reinterpret_cast<const Raw*>(p + 4 * i);
  }
  __device__ __forceinline__ void drop(int n) {
    if (n & 4) { q[0] = q[1]; q[1] = u32x4{0, 0, 0, 0}; }
    if (n & 2) { q[0] = u32x4{q[0][2], q[0][3], q[1][0], q[1][1]}; q[1] = u32x4{q[1][2], q[1][3], 0, 0}; }
    if (n & 1) { q[0] = u32x4{q[0][1], q[0][2], q[0][3], q[1][0]}; q[1] = u32x4{q[1][1], q[1][2], q[1][3], 0}; }
  }
  __device__ __forceinline__ void set(int c, float v) { q[c / 4][c % 4] = __float_as_uint(v); }
  __device__ __forceinline__ void clear() { q[0] = q[1] = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ float get(int c) const { return __uint_as_float(q[c / 4][c % 4]); }
  struct Top {
    unsigned m[8] = {};
    __device__ __forceinline__ void add(const Rows8& r) {
#pragma unroll
      for (int c = 0; c < 8; c++) {
        const unsigned a = r.q[c / 4][c % 4] & 0x7fffffffu;
        m[c] = a > m[c] ? a : m[c];
      }
    }
    __device__ __forceinline__ void across(int d) {
#pragma unroll
      for (int c = 0; c < 8; c++) {
        const unsigned a = (unsigned)__shfl_xor((int)m[c], d);
        m[c] = a > m[c] ? a : m[c];
      }
    }
    __device__ __forceinline__ unsigned get(int c) const { return m[c]; }
  };
};

template <typename T>
__global__ __launch_bounds__(512) void stash8_put_kernel(Stash8Slot p, const T* __restrict__ x, long ld) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];      // per wave 8 KiB of units; magnitudes and scales of the columns
  unsigned (*const top)[64] = reinterpret_cast<unsigned (*)[64]>(smem_raw + 8 * 8192);
  float* const scale_of = reinterpret_cast<float*>(smem_raw + 8 * 8192 + 8 * 256);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = tid & 7, rg = tid >> 3;
  const int c0 = (int)blockIdx.x * 64 + 8 * cg, block = (int)blockIdx.y, t0 = block * kStash8Block + 16 * rg;
  const int cn = p.cols - c0, tn = p.tokens - t0;  // columns and tokens from here on
  Rows8<T> v[16];
#pragma unroll
  for (int r = 0; r < 16; r++) v[r].clear();
  if (cn > 0 && tn > 0) {
    // (all loads before the first use of one, from the last row where there are no more: a load under a condition is waited for there)
    const int past = cn < 8 && p.cols >= 8 ? 8 - cn : 0;      // a row's last columns: the 8 that end there, without the first of them
    const T* const at = x + (long)t0 * ld + c0 - past;
    if (p.cols >= 8) {
#pragma unroll
      for (int r = 0; r < 16; r++) v[r].load(at + (long)(r < tn ? r : tn - 1) * ld);
      if (past) {
#pragma unroll
        for (int r = 0; r < 16; r++) v[r].drop(past);
      }
    } else {
#pragma unroll
      for (int r = 0; r < 16; r++)
#pragma unroll
        for (int c = 0; c < 8; c++) v[r].set(c, at[(long)(r < tn ? r : tn - 1) * ld + (c < cn ? c : cn - 1)]);
#pragma unroll
      for (int r = 0; r < 16; r++)
#pragma unroll
        for (int c = 0; c < 8; c++) if (c >= cn) v[r].set(c, (T)0.f);
    }
    if (tn < 16) {
#pragma unroll
      for (int r = 0; r < 16; r++) if (r >= tn) v[r].clear();
    }
  }
  typename Rows8<T>::Top m;
#pragma unroll
  for (int r = 0; r < 16; r++) m.add(v[r]);
#pragma unroll
  for (int d = 8; d < 64; d *= 2) m.across(d);
  if (lane < 8) {
#pragma unroll
    for (int c = 0; c < 8; c++) top[wave][8 * cg + c] = m.get(c);
  }
  __syncthreads();
  if (tid < 64) {
    unsigned a = 0;
#pragma unroll
    for (int w = 0; w < 8; w++) a = top[w][tid] > a ? top[w][tid] : a;
    // the largest value is f 2^k, 1 <= f < 2: in range with e = k - 6 where f <= 127 / 64
    int e = (int)(a >> 23) - 127 - 6 + ((a & 0x7fffffu) > 0x7e0000u);
    e = e < -126 ? -126 : e > kTopExponent ? kTopExponent : e;
    const float s = a < 0x7f800000u ? __uint_as_float((unsigned)(e + 127) << 23) : __builtin_nanf("");
    scale_of[tid] = s;
    const int c = (int)blockIdx.x * 64 + tid;
    if (c < 32 * p.col_blocks) p.scales[((long)p.slot * p.blocks + block) * 32 * p.col_blocks + c] = s;
  }
  __syncthreads();
  // The wave's 64 columns x 128 tokens are 8 halves of units, put together in LDS and stored as whole KiB (16 bytes at a time, spread over the lines, took
  // 35.4 us for 4096 x 11008, bf16).  Piece l of a half lies at l ^ (l / 8 % 8): the 8 lanes side by side write 128 bytes apart.
  unsigned char* const mine = smem_raw + wave * 8192;
  const int half = (cg >> 2) * 4 + ((rg & 7) >> 1), piece = 32 * (rg & 1) + 8 * (cg & 3);
#pragma unroll
  for (int c = 0; c < 8; c++) {
    const float s = scale_of[8 * cg + c];
    const bool fine = s == s;
    const float inv = fine ? __uint_as_float((254u << 23) - __float_as_uint(s)) : 0.f;      // 2^-e
    float x16[16];
#pragma unroll
    for (int r = 0; r < 16; r++) x16[r] = v[r].get(c);
    if (s == __uint_as_float((unsigned)(kTopExponent + 127) << 23)) {      // (rare: the one scale that values may pass the range of)
      const float most = 127.f * s;
#pragma unroll
      for (int r = 0; r < 16; r++) x16[r] = fminf(fmaxf(x16[r], -most), most);
    }
    u32x4 o;
#pragma unroll
    for (int q = 0; q < 4; q++) {
      // x 2^-e + 1.5 2^23, rounded once: the integer is in the low bits
      unsigned b[4];
#pragma unroll
      for (int i = 0; i < 4; i++) b[i] = __float_as_uint(__builtin_fmaf(x16[4 * q + i], inv, 12582912.f));
      const unsigned lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u);
      o[q] = fine ? lo | (hi << 16) : 0u;
    }
    *reinterpret_cast<u32x4*>(mine + half * 1024 + ((piece + c) ^ (piece >> 3)) * 16) = o;
  }
  // (LDS operations of a wave execute in order)
#pragma unroll
  for (int h = 0; h < 8; h++) {
    const int cb = 2 * (int)blockIdx.x + (h >> 2), t = block * kStash8Block + wave * 128 + 32 * (h & 3);
    if (cb < p.col_blocks && t < 64 * p.steps)
      *reinterpret_cast<u32x4*>(p.data + (((long)p.slot * p.steps + t / 64) * p.col_blocks + cb) * kUnit + (h & 1) * 1024 + lane * 16) =
          *reinterpret_cast<const u32x4*>(mine + h * 1024 + (lane ^ (lane >> 3)) * 16);
  }
}

// The way back: one thread = 16 tokens of 8 columns.  Bound by memory: 4096 x 11008 into bf16 21.9 us, 6.2 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void stash8_get_kernel(Stash8Slot p, T* __restrict__ y, long ld) {
  const int cg = threadIdx.x & 7, rg = (int)blockIdx.y * 32 + ((int)threadIdx.x >> 3);
  const int c0 = (int)blockIdx.x * 64 + 8 * cg, t0 = 16 * rg;
  if (c0 >= p.cols || t0 >= p.tokens) return;
  const unsigned char* const unit = p.data + (((long)p.slot * p.steps + t0 / 64) * p.col_blocks + c0 / 32) * kUnit + ((rg >> 1) & 1) * 1024 +
                                    (32 * (rg & 1) + c0 % 32) * 16;
  const float* const sc = p.scales + ((long)p.slot * p.blocks + t0 / kStash8Block) * 32 * p.col_blocks + c0;
  u32x4 q[8];
  float s[8];
#pragma unroll
  for (int c = 0; c < 8; c++) { q[c] = *reinterpret_cast<const u32x4*>(unit + 16 * c); s[c] = sc[c]; }      // (scales: up to the padded columns)
#pragma unroll
  for (int r = 0; r < 16; r++) {
    const int t = t0 + r;
    if (t >= p.tokens) break;
    float v[8];
#pragma unroll
    for (int c = 0; c < 8; c++) v[c] = (float)((int)(q[c][r / 4] << (24 - 8 * (r % 4))) >> 24) * s[c];
    T* const row = y + (long)t * ld + c0;
    if (p.cols - c0 >= 8) {
      typedef T Out __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));      // (any alignment, as above)
      constexpr int N = 16 / sizeof(T);
#pragma unroll
      for (int i = 0; i < 8; i += N) {
        Out o;
#pragma unroll
        for (int c = 0; c < N; c++) o[c] = (T)v[i + c];
        *reinterpret_cast<Out*>(row + i) = o;
      }
    } else {
      // a row's last columns: 4, 2 and 1 of them
      const int n = p.cols - c0;
      T* at = row;
      if (n & 4) {
        typedef T Four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
        *reinterpret_cast<Four*>(at) = Four{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
        at += 4;
      }
      const float a = n & 4 ? v[4] : v[0], b = n & 4 ? v[5] : v[1], c = n & 4 ? v[6] : v[2];
      if (n & 2) { at[0] = (T)a; at[1] = (T)b; at += 2; }
      if (n & 1) at[0] = (T)(n & 2 ? c : a);
    }
  }
}

// ------------------------------------------------------------------------------------------ dW = X^T dY
// Integers rather than 8-bit floats: on gfx950 the sums of 8-bit float products keep 13 bits below the largest of their group (1.5e-5 of the sums of N(0,1)
// products, measured), integer sums are whole; and a block's rounding of N(0,1) values is 1.0 % of them where e4m3 with the same kind of scale has 2.7 %.
// One workgroup = 4 waves, 2 x 2, each 32 MB x 32 NB of the output; the contraction in steps of 64 tokens through a ring of slots in LDS, filled by
// asynchronous copies all but one of them ahead.  The units are copied as they are: every fragment is 64 lanes x 16 bytes in a row.
// The integer sums of a block of tokens are exact: 1024 x 127^2 is below 2^24, so that they are exact in fp32 as well, in which the blocks are added
// up, each times the two columns' scales.  That takes three vector instructions per element and block, done tile by tile in front of the tile's first
// product of the next block (5 % of the time), and a second set of accumulators: 96 x 96 to a wave, one wave to a SIMD, or 64 x 64 and two.
// Bound by power on large outputs: 11008 x 4096 over 8 x 4096 tokens 1440 to 1720 us over cards, 1.72 to 2.05 PFLOP/s (at the rate of the bf16 weight gradients, 1.29, 2283), at 1.5 to 1.9 GHz with
// the matrix pipes busy 54 %; the same instructions on zeros take 7 % fewer cycles, at 2.27 GHz.  Rounds of few steps by their start and end (8 us): 4096 x 4096 over 4096
// tokens 80 us, 1.7 PFLOP/s.  Tried without gain: copies spread over all of a step's products; tiles of 128 x 96 and 128 x 64 to a wave (1594 and 1653 us for 1588).
constexpr int dw_slots(int mb, int nb, int per_cu) { return (160 * 1024 / per_cu - 8 * 2048) / (2 * (mb + nb) * kUnit); }
struct Stash8Dw {
  const unsigned char* x; const float* xs; int xb;     // units, scales, column blocks
  const unsigned char* dy; const float* ds; int db;
  float* dw; long ld;
  int M, N, accumulate;
  int steps, blocks;                                   // of a slot
  long first_step, first_block;                        // of the run
  int total;                                           // steps of the run
  int tiles_m, tiles_n;
  int shares, share;                                   // of the contraction: how many, and blocks of each but the last
  float* part;                                         // shares > 1: [share][tile][wave][tile of 32 x 32][quarter][lane][4], as the accumulators lie
};

template <int MB, int NB, int PER_CU>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(PER_CU, PER_CU))) void stash8_dw_kernel(Stash8Dw p) {
  constexpr int WM = 2, WN = 2;
  constexpr int UA = MB * WM, UB = NB * WN;            // units of a step
  constexpr int SLOT = (UA + UB) * kUnit, SLOTS = dw_slots(MB, NB, PER_CU), AHEAD = SLOTS - 1;
  constexpr int OPS = 2 * (UA + UB) / 4;               // copies of a step, per wave
  static_assert(2 * UA % 4 == 0 && 2 * UB % 4 == 0 && UA <= 8 && UB <= 8, "copies are shared out evenly");
  constexpr int SCALES = 512 * 4, RING = 8;            // 256 scales of x, 256 of dy; as many blocks may be under way as steps, and one in use
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  lds_u8* const lds = LDS_PTR(unsigned char, smem_raw);
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds, sc0 = lds0 + SLOTS * SLOT;
  lds_u8* const sc = lds + SLOTS * SLOT;

  const int lane = threadIdx.x & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  // tiles: ids go round the 8 XCDs; each gets a run of them, walked in bands of 4 rows, so that what an XCD works on at a time shares operands in its cache
  int tm, tn;
  {
    const int tiles = p.tiles_m * p.tiles_n, id = (int)blockIdx.x % tiles, per = tiles / 8, rest = tiles % 8;
    const int xcd = id % 8, at = id / 8;
    const int t = xcd * per + (xcd < rest ? xcd : rest) + at;
    const int band = t / (4 * p.tiles_n), in = t - band * 4 * p.tiles_n;
    const int rows = p.tiles_m - 4 * band < 4 ? p.tiles_m - 4 * band : 4;
    tn = in / rows;
    tm = 4 * band + in - tn * rows;
  }
  // the share's steps: whole blocks, so that their integer sums stay whole
  const int share = (int)blockIdx.x / (p.tiles_m * p.tiles_n);
  auto step_of = [&](long b) {                         // at which the run's block b begins
    const long slot = b / p.blocks;
    const long s = slot * p.steps + (b - slot * p.blocks) * kStepsPerBlock;
    return (int)(s < p.total ? s : p.total);
  };
  const int s0 = step_of((long)share * p.share), total = step_of((long)(share + 1) * p.share) - s0;
  // block -1, which is added before the first one
  for (int i = (int)threadIdx.x; i < SCALES / 4; i += 256) reinterpret_cast<LDS_AS float*>(sc + (RING - 1) * SCALES)[i] = 0.f;
  const int ub_a = tm * UA, ub_b = tn * UB;            // first column blocks
  const int na = p.xb - ub_a < UA ? p.xb - ub_a : UA, nb = p.db - ub_b < UB ? p.db - ub_b : UB;

  // The copies of a step into its slot, in order from step 0 on: chunks of 1 KiB, x's units first; chunks past the last column block, and steps past the last one,
  // deliver zeros.  begin() sets up the next step's, copy(i) issues the wave's i-th.
  const long step0 = p.first_step + s0, block0 = p.first_block + (long)share * p.share;
  const int in = s0 % p.steps;                         // steps of its slot before the share's first
  const unsigned char* at_a = p.x + (step0 * p.xb + ub_a) * kUnit;
  const unsigned char* at_b = p.dy + (step0 * p.db + ub_b) * kUnit;
  const float* at_sa = p.xs + (block0 * p.xb + ub_a) * 32;
  const float* at_sb = p.ds + (block0 * p.db + ub_b) * 32;
  const long next_a = (long)p.xb * kUnit, next_b = (long)p.db * kUnit;
  int to_come = total, in_slot = in;                   // steps to be copied; of the next one: steps since the slot's first, and since the block's
  int in_block = 0;
  uint32_t slot_w = lds0 + wave * 1024, scale_w = sc0 + wave * 256;
  u32x4 da, db;
  auto begin = [&] {
    const bool live = to_come > 0;
    da = make_desc(at_a, live ? na * kUnit : 0);
    db = make_desc(at_b, live ? nb * kUnit : 0);
    if (in_block == 0) {                               // the scales of the block that begins
      const u32x4 sa = make_desc(at_sa, live ? na * 128 : 0), sb = make_desc(at_sb, live ? nb * 128 : 0);
      dma4(scale_w, sa, wave * 256 + lane * 4);
      dma4(scale_w + 1024, sb, wave * 256 + lane * 4);
      at_sa += p.xb * 32;
      at_sb += p.db * 32;
      scale_w = scale_w + SCALES >= sc0 + RING * SCALES ? sc0 + wave * 256 : scale_w + SCALES;
    }
  };
  const uint32_t voff = wave * 1024 + lane * 16;
  auto copy = [&](int i) {
    if (4 * i < 2 * UA) dma16(slot_w + i * 4096, da, voff + i * 4096);
    else dma16(slot_w + i * 4096, db, voff + i * 4096 - 2 * UA * 1024);
  };
  auto done = [&] {
    at_a += next_a;
    at_b += next_b;
    to_come--;
    slot_w = slot_w + SLOT >= lds0 + SLOTS * SLOT ? lds0 + wave * 1024 : slot_w + SLOT;
    in_block = in_block + 1 == kStepsPerBlock ? 0 : in_block + 1;
    if (++in_slot == p.steps) { in_slot = 0; in_block = 0; }
  };

  i32x16 ia[MB][NB];
  f32x16 fa[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; i++)
#pragma unroll
    for (int j = 0; j < NB; j++)
#pragma unroll
      for (int e = 0; e < 16; e++) { fa[i][j][e] = 0.f; ia[i][j][e] = 0; }

  // Fragments of a half step: first the first tile's, then those of its row and column.
  i32x4 fra[2][MB], frb[2][NB];
  lds_u8* const mine = lds + lane * 16;
  auto fetch = [&](int to, int slot, int half, int k) {
    lds_u8* const from = mine + slot + half * 1024;
    if (k == 0) frb[to][0] = *reinterpret_cast<LDS_AS const i32x4*>(from + (UA + wn * NB) * kUnit);
    else if (k == 1) fra[to][0] = *reinterpret_cast<LDS_AS const i32x4*>(from + wm * MB * kUnit);
    else if (k < NB + 1) frb[to][k - 1] = *reinterpret_cast<LDS_AS const i32x4*>(from + (UA + wn * NB + k - 1) * kUnit);
    else fra[to][k - NB] = *reinterpret_cast<LDS_AS const i32x4*>(from + (wm * MB + k - NB) * kUnit);
  };
  // What the block's integer sums add to the result: a tile, by the scales of its rows and of the lane's column.  The integer takes the column's first and the row's
  // as the rounded sum is formed: the product of the two scales may be infinite where the integer is 0, or too small for fp32 where the result is not.  Below 2^24,
  // the integer times a scale up to 2^103 is exact and finite.  Of a larger one (`high`: some column of the wave's has one) 2^24 goes to the rows, but for
  // those above 2^103 themselves, with which the result is 0 or infinite all the same.
  constexpr float HIGH = 0x1p103f;
  f32x4 sa[4];
  float sb[NB];
  bool high = false, moved[NB];
  auto rows_of = [&](int i, int block) {
    const LDS_AS float* const s = reinterpret_cast<const LDS_AS float*>(sc + (block & (RING - 1)) * SCALES);
#pragma unroll
    for (int q = 0; q < 4; q++) sa[q] = *reinterpret_cast<const LDS_AS f32x4*>(s + 32 * (wm * MB + i) + 8 * q + 4 * g);
  };
  auto scales_of = [&](int i, int block) {
    if (i == 0) {
      const LDS_AS float* const s = reinterpret_cast<const LDS_AS float*>(sc + (block & (RING - 1)) * SCALES);
      bool any = false;
#pragma unroll
      for (int j = 0; j < NB; j++) {
        const float b = s[256 + 32 * (wn * NB + j) + (lane & 31)];
        moved[j] = b > HIGH;
        sb[j] = moved[j] ? b * 0x1p-24f : b;
        any |= moved[j];
      }
      high = __any(any);
    }
    rows_of(i, block);
  };
  auto add_tile = [&](int i, int j, int block) {
    if (__builtin_expect(high, 0)) {
      rows_of(i, block);
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const float row = sa[e >> 2][e & 3];
        sa[e >> 2][e & 3] = moved[j] && !(row > HIGH) ? row * 0x1p24f : row;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; e++) fa[i][j][e] = __builtin_fmaf((float)ia[i][j][e] * sb[j], sa[e >> 2][e & 3], fa[i][j][e]);
    asm volatile("" : "+v"(fa[i][j]));                // (here and now: the compiler would keep all the integers for later)
  };

  // One step, in a pinned order (the compiler would put each fragment's read right before its product): the second half's fragments are fetched beside the products
  // of the first, the next step's first half beside those of the second, and copies issued there.
  // BEGIN: the block's first step, whose products start from zero, and in front of each of them the tile's sums of the block before.
  int slot_r = 0;
  auto step = [&](auto is_first, int before) {
    constexpr bool BEGIN = decltype(is_first)::value;
    // step s + 1 has landed (no more than the copies of the steps behind it are under way, or fewer, where scales are among them); every wave is done with step s - 1
    wait_vmem<(AHEAD - 2) * OPS>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int next_r = slot_r + SLOT == SLOTS * SLOT ? 0 : slot_r + SLOT;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < MB * NB; k++) {
      const int i = k / NB, j = k % NB;
      if constexpr (BEGIN) {
        if (j == 0) scales_of(i, before);
        add_tile(i, j, before);
#pragma unroll
        for (int e = 0; e < 16; e++) ia[i][j][e] = 0;
      }
      ia[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fra[0][i], frb[0][j], ia[i][j], 0, 0, 0);
      if (k < MB + NB) fetch(1, slot_r, 1, k);
      if (k == MB * NB - 1) begin();
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int k = 0; k < MB * NB; k++) {
      const int i = k / NB, j = k % NB;
      ia[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fra[1][i], frb[1][j], ia[i][j], 0, 0, 0);
      if (k < MB + NB) fetch(0, next_r, 0, k);
      if (k < OPS) copy(k);
      if (k == MB * NB - 1) done();
      __builtin_amdgcn_sched_barrier(0);
    }
    slot_r = next_r;
  };
  static_assert(OPS <= MB * NB && MB + NB <= MB * NB, "a step's copies and fragments beside its products");
  for (int i = 0; i < AHEAD; i++) {
    begin();
#pragma unroll
    for (int k = 0; k < OPS; k++) copy(k);
    done();
  }
  wait_vmem<0>();
  __syncthreads();
#pragma unroll
  for (int k = 0; k < MB + NB; k++) fetch(0, 0, 0, k);
  int block = 0, left = p.steps - in;                  // blocks since the share's first; steps left of the slot
  for (int s = 0; s < total; block++) {
    const int n = left < kStepsPerBlock ? left : kStepsPerBlock;
    step(std::true_type(), block - 1);                 // (before the first block: zeros, by scales that are zeros)
    for (int i = 1; i < n; i++) step(std::false_type(), 0);
    s += n;
    left = left == n ? p.steps : left - n;
  }
  wait_vmem<0>();                                      // (copies past the end: zeros)
  if (MB == 2 && p.shares > 1) {                       // (only the small tiles are so few)
    f32x4* const part = reinterpret_cast<f32x4*>(p.part) + (((long)share * p.tiles_m * p.tiles_n + (long)tm * p.tiles_n + tn) * 4 + wave) * (MB * NB * 256) + lane;
#pragma unroll
    for (int i = 0; i < MB; i++) {
      scales_of(i, block - 1);
#pragma unroll
      for (int j = 0; j < NB; j++) {
        add_tile(i, j, block - 1);
#pragma unroll
        for (int q = 0; q < 4; q++) part[((i * NB + j) * 4 + q) * 64] = f32x4{fa[i][j][4 * q], fa[i][j][4 * q + 1], fa[i][j][4 * q + 2], fa[i][j][4 * q + 3]};
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < MB; i++) {
    scales_of(i, block - 1);
#pragma unroll
    for (int j = 0; j < NB; j++) {
      add_tile(i, j, block - 1);
      const int n = 32 * (ub_b + wn * NB + j) + (lane & 31);
      if (n < p.N) {
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int m = 32 * (ub_a + wm * MB + i) + 8 * (e >> 2) + 4 * g + (e & 3);
          if (m < p.M) {
            float* const o = p.dw + (long)m * p.ld + n;
            *o = p.accumulate ? *o + fa[i][j][e] : fa[i][j][e];
          }
        }
      }
    }
  }
}

// The shares of a tile, added up in order: a thread has 4 elements of every share.
template <int MB, int NB>
__global__ __launch_bounds__(256) void stash8_join_kernel(Stash8Dw p) {
  const long tiles = (long)p.tiles_m * p.tiles_n;
  const int tile = (int)blockIdx.x / (MB * NB * 4), in = (int)blockIdx.x % (MB * NB * 4);      // 256 of a tile's 4 x MB NB x 256 threads
  const int wave = in / (MB * NB), t = in % (MB * NB), lane = (int)threadIdx.x & 63, q = (int)threadIdx.x >> 6;
  const int tm = tile / p.tiles_n, tn = tile - tm * p.tiles_n;
  const int m = 32 * (tm * 2 * MB + (wave >> 1) * MB + t / NB) + 8 * q + 4 * (lane >> 5), n = 32 * (tn * 2 * NB + (wave & 1) * NB + t % NB) + (lane & 31);
  if (n >= p.N || m >= p.M) return;
  const f32x4* const part = reinterpret_cast<const f32x4*>(p.part) + (tile * 4L + wave) * (MB * NB * 256) + (t * 4 + q) * 64 + lane;
  f32x4 v = part[0];
  for (int s = 1; s < p.shares; s++) v += part[s * tiles * 4 * (MB * NB * 256)];
#pragma unroll
  for (int e = 0; e < 4; e++)
    if (m + e < p.M) {
      float* const o = p.dw + (long)(m + e) * p.ld + n;
      *o = p.accumulate ? *o + v[e] : v[e];
    }
}

// ------------------------------------------------------------------------------------------ launches
template <typename T>
static hipError_t launch_put(const Stash8Slot& p, const void* x, long ld, hipStream_t s) {
  constexpr size_t smem = 8 * 8192 + 8 * 256 + 256;
  auto kern = stash8_put_kernel<T>;
  static AttrOnce once;
  if (hipError_t e = once.set(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)((p.cols + 63) / 64), (unsigned)p.blocks), dim3(512), smem, s, p, (const T*)x, ld);
  return hipGetLastError();
}

hipError_t stash8_put(int dtype, const Stash8Slot& p, const void* x, long ld, hipStream_t s) {
  return dtype ? launch_put<bf16_t>(p, x, ld, s) : launch_put<float>(p, x, ld, s);
}

hipError_t stash8_get(int dtype, const Stash8Slot& p, void* y, long ld, hipStream_t s) {
  const dim3 grid((unsigned)((p.cols + 63) / 64), (unsigned)((p.tokens + 511) / 512)), block(256);
  if (dtype) hipLaunchKernelGGL(stash8_get_kernel<bf16_t>, grid, block, 0, s, p, (bf16_t*)y, ld);
  else hipLaunchKernelGGL(stash8_get_kernel<float>, grid, block, 0, s, p, (float*)y, ld);
  return hipGetLastError();
}

// Tiles of 96 x 96 to a wave and one workgroup to a compute unit, or of 64 x 64 and two, by the time that their rounds of workgroups take: us per step and
// per round.  Measured, 96 / 64: 11008 x 4096 over 8 x 4096 tokens 1702 / 1780, 5120 x 13824 over 4 x 4096 1204 / 1259, 8 x 1024 4096 x 11008 398 / 393, 4096 x 4096 over 8 x
// 4096 570 / 560, 12288 x 4096 over 2 x 1024 173 / 134.
// Shares of the contraction where there are few tiles, each of whole blocks, three at least.  us, one / shares: 512 x 512 over 8 x 2048 tokens 75 / 20, 1536 x 1536 over 8 x 4096 143 /
// 98, 2048 x 1024 over 4 x 4096 77 / 50, but 2048 x 2048 over 8 x 1024 in two 48 / 51.
Stash8Plan stash8_plan(int m, int n, int steps, int blocks) {
  const long mb = (m + 31) / 32, nb = (n + 31) / 32;
  const long large = ((mb + 5) / 6) * ((nb + 5) / 6), small = ((mb + 3) / 4) * ((nb + 3) / 4);
  const float of_large = (float)((large + 255) / 256) * (0.603f * steps + 9.f), rest = (float)(small % 512);
  const float of_small = (float)(small / 512) * (0.524f * steps + 8.f) + (rest ? (rest <= 256 ? 0.4f : 0.524f) * steps + 8.f : 0.f);
  if (large >= 256 && of_large < of_small) return Stash8Plan{3, 3, 1, blocks, 0};
  Stash8Plan r{2, 2, 1, blocks, 0};
  long shares = 512 / small;
  shares = shares < steps / 4 ? shares : steps / 4;
  shares = shares < blocks ? shares : blocks;
  if (shares >= 3) {
    r.share = (int)((blocks + shares - 1) / shares);
    r.shares = (blocks + r.share - 1) / r.share;
    r.bytes = (size_t)r.shares * small * 128 * 128 * sizeof(float);
  }
  return r;
}

template <int MB, int NB, int PER_CU>
static hipError_t launch_dw(Stash8Dw p, hipStream_t s) {
  constexpr size_t smem = dw_slots(MB, NB, PER_CU) * (2 * MB + 2 * NB) * kUnit + 8 * 2048;
  auto kern = stash8_dw_kernel<MB, NB, PER_CU>;
  static AttrOnce once;
  if (hipError_t e = once.set(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  p.tiles_m = (p.xb + 2 * MB - 1) / (2 * MB);
  p.tiles_n = (p.db + 2 * NB - 1) / (2 * NB);
  const long tiles = (long)p.tiles_m * p.tiles_n;
  hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * p.shares)), dim3(256), smem, s, p);
  if constexpr (MB == 2)
    if (p.shares > 1) hipLaunchKernelGGL((stash8_join_kernel<MB, NB>), dim3((unsigned)(tiles * MB * NB * 4)), dim3(256), 0, s, p);
  return hipGetLastError();
}

hipError_t stash8_dw(const Stash8Slot& x, const Stash8Slot& dy, int n, float* dw, long ld, int accumulate, float* part, hipStream_t s) {
  Stash8Dw p{};
  p.x = x.data; p.xs = x.scales; p.xb = x.col_blocks; p.dy = dy.data; p.ds = dy.scales; p.db = dy.col_blocks;
  p.dw = dw; p.ld = ld; p.M = x.cols; p.N = dy.cols; p.accumulate = accumulate;
  p.steps = x.steps; p.blocks = x.blocks;
  p.first_step = (long)x.slot * x.steps; p.first_block = (long)x.slot * x.blocks; p.total = n * x.steps;
  const Stash8Plan plan = stash8_plan(x.cols, dy.cols, p.total, n * x.blocks);
  p.shares = plan.shares; p.share = plan.share; p.part = part;
  return plan.mb == 3 ? launch_dw<3, 3, 1>(p, s) : launch_dw<2, 2, 2>(p, s);
}

}  // namespace tbp
