// A stash in 8 bits for gfx950: a linear layer's inputs and output derivatives are kept from backward-p1 to backward-p2 as 8-bit integers,
// and the weight gradient dW = X^T dY is formed from them on the integer matrix instructions.
//
// Of every kStash8Block tokens of a column (counted from a slot's first token) the values are q 2^e with q = -127 .. 127 and e the smallest exponent,
// -126 at least, with which the largest of them is in that range (121 at most: beyond, q ends at 127); q is the nearest integer, halves to even.  Powers of two, so that scaling is exact and
// the one rounding is q's: at most half of 2^e, which is at most 2^-6 of the block's largest value.
// A block that holds an infinity or a NaN has no such scale: its scale is NaN, and with it all that it stands for.
//
// Layout: the matrix instructions want, per column, consecutive tokens.  A unit of 32 columns x 64 tokens is 2 KiB: two halves of 32 tokens, in each the
// 16 bytes of lane l = tokens 16 (l / 32) .. of column l % 32, as the instruction's operand lies in its registers.  Units lie column block after column
// block, then 64 tokens after 64 tokens, then slot after slot (a slot's tokens are padded with zeros to a multiple of 64), so that the slots of a step are
// one contraction length.  Behind them the scales, fp32: [slot][block of tokens][column].
#include "kernels.h"
#include "rows.h"

namespace tbp {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kUnit = 2048;                      // bytes of a unit
constexpr int kStepsPerBlock = kStash8Block / 64;
constexpr int kTopExponent = 121;                // of a scale: 127 2^121 is the largest multiple that fp32 has

// ------------------------------------------------------------------------------------------ into the stash, and out of it
// One workgroup = 64 columns of one block of tokens, 8 threads side by side with 8 columns each (128 bytes of a row, bf16) and 64 of them below each other
// with 16 tokens each, which stay in registers between the two looks at them: the largest magnitude of every column, then the rounding.
// Magnitudes are compared as bit patterns, in which NaN is above infinity.
template <typename T, bool WIDE>
__global__ __launch_bounds__(512) void stash8_put_kernel(Stash8Slot p, const T* __restrict__ x, long ld) {
  __shared__ unsigned top[8][64];
  __shared__ float scale_of[64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = tid & 7, rg = tid >> 3;
  const int c0 = (int)blockIdx.x * 64 + 8 * cg, block = (int)blockIdx.y, t0 = block * kStash8Block + 16 * rg;
  float v[16][8];
  const int cn = p.cols - c0;                      // columns from here on
#pragma unroll
  for (int r = 0; r < 16; r++) {
    const int t = t0 + r;
    const T* const row = x + (long)t * ld + c0;
    if (WIDE && t < p.tokens && cn >= 8) {
      if constexpr (sizeof(T) == 2) Vec<bf16_t>::load(row, v[r]);
      else { Vec<float>::load(row, v[r]); Vec<float>::load(row + 4, v[r] + 4); }
    } else {
#pragma unroll
      for (int c = 0; c < 8; c++) v[r][c] = t < p.tokens && c < cn ? (float)row[c] : 0.f;
    }
  }
  unsigned m[8];
#pragma unroll
  for (int c = 0; c < 8; c++) {
    m[c] = 0;
#pragma unroll
    for (int r = 0; r < 16; r++) {
      const unsigned a = __float_as_uint(v[r][c]) & 0x7fffffffu;
      m[c] = a > m[c] ? a : m[c];
    }
#pragma unroll
    for (int d = 8; d < 64; d *= 2) {
      const unsigned a = (unsigned)__shfl_xor((int)m[c], d);
      m[c] = a > m[c] ? a : m[c];
    }
  }
  if (lane < 8) {
#pragma unroll
    for (int c = 0; c < 8; c++) top[wave][8 * cg + c] = m[c];
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
  if (c0 >= 32 * p.col_blocks || t0 >= 64 * p.steps) return;
  unsigned char* const unit = p.data + (((long)p.slot * p.steps + t0 / 64) * p.col_blocks + c0 / 32) * kUnit + ((rg >> 1) & 1) * 1024 +
                              (32 * (rg & 1) + c0 % 32) * 16;
#pragma unroll
  for (int c = 0; c < 8; c++) {
    const float s = scale_of[8 * cg + c];
    const bool fine = s == s;
    const float inv = fine ? __uint_as_float((254u << 23) - __float_as_uint(s)) : 0.f;      // 2^-e
    if (s == __uint_as_float((unsigned)(kTopExponent + 127) << 23)) {      // (rare: the one scale that values may pass the range of)
      const float most = 127.f * s;
#pragma unroll
      for (int r = 0; r < 16; r++) v[r][c] = fminf(fmaxf(v[r][c], -most), most);
    }
    u32x4 o;
#pragma unroll
    for (int q = 0; q < 4; q++) {
      // x 2^-e + 1.5 2^23, rounded once: the integer is in the low bits
      unsigned b[4];
#pragma unroll
      for (int i = 0; i < 4; i++) b[i] = __float_as_uint(__builtin_fmaf(v[4 * q + i][c], inv, 12582912.f));
      const unsigned lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u);
      o[q] = fine ? lo | (hi << 16) : 0u;
    }
    *reinterpret_cast<u32x4*>(unit + 16 * c) = o;
  }
}

// The way back: one thread = 16 tokens of 8 columns.
template <typename T, bool WIDE>
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
    if (WIDE && p.cols - c0 >= 8) {
      if constexpr (sizeof(T) == 2) Vec<bf16_t>::store(row, v);
      else { Vec<float>::store(row, v); Vec<float>::store(row + 4, v + 4); }
    } else {
#pragma unroll
      for (int c = 0; c < 8; c++)
        if (c < p.cols - c0) row[c] = (T)v[c];
    }
  }
}

// ------------------------------------------------------------------------------------------ dW = X^T dY
// One workgroup = 4 waves, 2 x 2, each 128 x 32 NB of the output; the contraction in steps of 64 tokens through a ring of four slots in LDS, filled by
// asynchronous copies three steps ahead.  The units are copied as they are: every fragment is 64 lanes x 16 bytes in a row.
// The integer sums of a block of tokens are exact: 1024 x 127^2 is below 2^24, so that they are exact in fp32 as well, in which the blocks are added
// up, each with the product of the two columns' scales.  That takes three vector instructions per element and block, done tile by tile in front of the tile's first
// product of the next block, and a second set of accumulators, which one wave per SIMD has the registers for.
struct Stash8Dw {
  const unsigned char* x; const float* xs; int xb;     // units, scales, column blocks
  const unsigned char* dy; const float* ds; int db;
  float* dw; long ld;
  int M, N, accumulate;
  int steps, blocks;                                   // of a slot
  long first_step, first_block;                        // of the run
  int total;                                           // steps of the run
  int tiles_m, tiles_n;
};

template <int MB, int NB>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) void stash8_dw_kernel(Stash8Dw p) {
  constexpr int WM = 2, WN = 2;
  constexpr int UA = MB * WM, UB = NB * WN;            // units of a step
  constexpr int SLOT = (UA + UB) * kUnit, SLOTS = 4;
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
    const int tiles = p.tiles_m * p.tiles_n, id = (int)blockIdx.x, per = tiles / 8, rest = tiles % 8;
    const int xcd = id % 8, at = id / 8;
    const int t = xcd * per + (xcd < rest ? xcd : rest) + at;
    const int band = t / (4 * p.tiles_n), in = t - band * 4 * p.tiles_n;
    const int rows = p.tiles_m - 4 * band < 4 ? p.tiles_m - 4 * band : 4;
    tn = in / rows;
    tm = 4 * band + in - tn * rows;
  }
  const int ub_a = tm * UA, ub_b = tn * UB;            // first column blocks
  const int na = p.xb - ub_a < UA ? p.xb - ub_a : UA, nb = p.db - ub_b < UB ? p.db - ub_b : UB;

  // The copies of step s into its slot: chunks of 1 KiB, x's units first; chunks past the last column block, and steps past the last one, deliver zeros.
  int at_block = 0, in_block = 0, in_slot = 0;         // of the next step to be copied: blocks since the run's first, steps since the block's and the slot's first
  auto issue = [&](int s) {
    const bool live = s < p.total;
    const long step = p.first_step + (live ? s : 0);
    const u32x4 da = make_desc(p.x + (step * p.xb + ub_a) * kUnit, live ? na * kUnit : 0);
    const u32x4 db = make_desc(p.dy + (step * p.db + ub_b) * kUnit, live ? nb * kUnit : 0);
    const uint32_t slot = lds0 + (s % SLOTS) * SLOT;
#pragma unroll
    for (int i = 0; i < OPS; i++) {
      const int chunk = wave + 4 * i;                  // (uniform)
      if (4 * i < 2 * UA) dma16(slot + chunk * 1024, da, chunk * 1024 + lane * 16);
      else dma16(slot + chunk * 1024, db, (chunk - 2 * UA) * 1024 + lane * 16);
    }
    if (in_block == 0) {                               // the scales of the block that begins
      const long b = p.first_block + at_block;
      const u32x4 sa = make_desc(p.xs + (b * p.xb + ub_a) * 32, live ? na * 128 : 0);
      const u32x4 sb = make_desc(p.ds + (b * p.db + ub_b) * 32, live ? nb * 128 : 0);
      const uint32_t to = sc0 + (at_block % RING) * SCALES + wave * 256;
      dma4(to, sa, wave * 256 + lane * 4);
      dma4(to + 1024, sb, wave * 256 + lane * 4);
    }
    in_block++;
    if (++in_slot == p.steps) { in_slot = 0; in_block = 0; at_block++; }
    else if (in_block == kStepsPerBlock) { in_block = 0; at_block++; }
  };

  i32x16 ia[MB][NB];
  f32x16 fa[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; i++)
#pragma unroll
    for (int j = 0; j < NB; j++)
#pragma unroll
      for (int e = 0; e < 16; e++) { fa[i][j][e] = 0.f; ia[i][j][e] = 0; }

  i32x4 fra[2][MB], frb[2][NB];
  auto fetch = [&](int to, int s, int half) {
    lds_u8* const slot = lds + (s % SLOTS) * SLOT + half * 1024 + lane * 16;
#pragma unroll
    for (int i = 0; i < MB; i++) fra[to][i] = *reinterpret_cast<LDS_AS const i32x4*>(slot + (wm * MB + i) * kUnit);
#pragma unroll
    for (int j = 0; j < NB; j++) frb[to][j] = *reinterpret_cast<LDS_AS const i32x4*>(slot + (UA + wn * NB + j) * kUnit);
  };
  // what the block's integer sums add to the result: tile row i
  auto add_block = [&](int i, int block) {
    const LDS_AS float* const s = reinterpret_cast<const LDS_AS float*>(sc + (block % RING) * SCALES);
    f32x4 sa[4];
#pragma unroll
    for (int q = 0; q < 4; q++) sa[q] = *reinterpret_cast<const LDS_AS f32x4*>(s + 32 * (wm * MB + i) + 8 * q + 4 * g);
#pragma unroll
    for (int j = 0; j < NB; j++) {
      const float sb = s[256 + 32 * (wn * NB + j) + (lane & 31)];
#pragma unroll
      for (int e = 0; e < 16; e++) fa[i][j][e] = __builtin_fmaf((float)ia[i][j][e], sa[e >> 2][e & 3] * sb, fa[i][j][e]);
    }
  };

  // first steps of blocks among the next to be waited for
  auto begins = [&](int step_in_slot) { return step_in_slot % kStepsPerBlock == 0; };
  issue(0);
  issue(1);
  issue(2);
  wait_vmem<0>();
  __syncthreads();
  fetch(0, 0, 0);
  int block = -1, here = 0, ahead = 2 % p.steps;       // the block in work; steps since the slot's first, of this step and of the one after next
  for (int s = 0; s < p.total; s++) {
    // step s + 1 has landed (only step s + 2 may still be under way); every wave is done with step s - 1
    if (begins(ahead)) wait_vmem<OPS + 2>(); else wait_vmem<OPS>();
    __syncthreads();
    issue(s + 3);
    fetch(1, s, 1);
    if (begins(here)) {
#pragma unroll
      for (int i = 0; i < MB; i++) {
        if (block >= 0) add_block(i, block);
#pragma unroll
        for (int j = 0; j < NB; j++) {
          i32x16 z;
#pragma unroll
          for (int e = 0; e < 16; e++) z[e] = 0;
          ia[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fra[0][i], frb[0][j], z, 0, 0, 0);
        }
      }
      block++;
    } else {
#pragma unroll
      for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++) ia[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fra[0][i], frb[0][j], ia[i][j], 0, 0, 0);
    }
    fetch(0, s + 1, 0);
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
      for (int j = 0; j < NB; j++) ia[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fra[1][i], frb[1][j], ia[i][j], 0, 0, 0);
    if (++here == p.steps) here = 0;
    if (++ahead == p.steps) ahead = 0;
  }
  wait_vmem<0>();                                      // (copies past the end: zeros)
#pragma unroll
  for (int i = 0; i < MB; i++) {
    if (block >= 0) add_block(i, block);
#pragma unroll
    for (int j = 0; j < NB; j++) {
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

// ------------------------------------------------------------------------------------------ launches
hipError_t stash8_put(int dtype, const Stash8Slot& p, const void* x, long ld, hipStream_t s) {
  const dim3 grid((unsigned)((p.cols + 63) / 64), (unsigned)p.blocks), block(512);
  const bool wide = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld % (dtype ? 8 : 4) == 0;
  if (dtype) {
    if (wide) hipLaunchKernelGGL((stash8_put_kernel<bf16_t, true>), grid, block, 0, s, p, (const bf16_t*)x, ld);
    else hipLaunchKernelGGL((stash8_put_kernel<bf16_t, false>), grid, block, 0, s, p, (const bf16_t*)x, ld);
  } else {
    if (wide) hipLaunchKernelGGL((stash8_put_kernel<float, true>), grid, block, 0, s, p, (const float*)x, ld);
    else hipLaunchKernelGGL((stash8_put_kernel<float, false>), grid, block, 0, s, p, (const float*)x, ld);
  }
  return hipGetLastError();
}

hipError_t stash8_get(int dtype, const Stash8Slot& p, void* y, long ld, hipStream_t s) {
  const dim3 grid((unsigned)((p.cols + 63) / 64), (unsigned)((p.tokens + 511) / 512)), block(256);
  const bool wide = reinterpret_cast<uintptr_t>(y) % 16 == 0 && ld % (dtype ? 8 : 4) == 0;
  if (dtype) {
    if (wide) hipLaunchKernelGGL((stash8_get_kernel<bf16_t, true>), grid, block, 0, s, p, (bf16_t*)y, ld);
    else hipLaunchKernelGGL((stash8_get_kernel<bf16_t, false>), grid, block, 0, s, p, (bf16_t*)y, ld);
  } else {
    if (wide) hipLaunchKernelGGL((stash8_get_kernel<float, true>), grid, block, 0, s, p, (float*)y, ld);
    else hipLaunchKernelGGL((stash8_get_kernel<float, false>), grid, block, 0, s, p, (float*)y, ld);
  }
  return hipGetLastError();
}

template <int MB, int NB>
static hipError_t launch_dw(Stash8Dw p, hipStream_t s) {
  constexpr size_t smem = 4 * (2 * MB + 2 * NB) * kUnit + 8 * 2048;
  auto kern = stash8_dw_kernel<MB, NB>;
  static AttrOnce once;
  if (hipError_t e = once.set(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  p.tiles_m = (p.xb + 2 * MB - 1) / (2 * MB);
  p.tiles_n = (p.db + 2 * NB - 1) / (2 * NB);
  hipLaunchKernelGGL(kern, dim3((unsigned)(p.tiles_m * p.tiles_n)), dim3(256), smem, s, p);
  return hipGetLastError();
}

hipError_t stash8_dw(const Stash8Slot& x, const Stash8Slot& dy, int n, float* dw, long ld, int accumulate, hipStream_t s) {
  Stash8Dw p{};
  p.x = x.data; p.xs = x.scales; p.xb = x.col_blocks; p.dy = dy.data; p.ds = dy.scales; p.db = dy.col_blocks;
  p.dw = dw; p.ld = ld; p.M = x.cols; p.N = dy.cols; p.accumulate = accumulate;
  p.steps = x.steps; p.blocks = x.blocks;
  p.first_step = (long)x.slot * x.steps; p.first_block = (long)x.slot * x.blocks; p.total = n * x.steps;
  if (0) return launch_dw<4, 2>(p, s);
  return launch_dw<3, 3>(p, s);
}

}  // namespace tbp
