// Sliding-window attention with sinks for gfx950 (bf16 storage, fp32 accumulation, head_dim 64 or 128, grouped heads): forward,
// backward-p1, and the form for one new token per sequence over a cache; forward and backward-p1 also over packed sequences, causal without a window.
//
// Query i of a sequence of n tokens sees key j when j <= i and (j > i - window or j < sinks); tokens n .. S - 1 of a row of the
// batch are padding: never read, zeros in every result (lse: -inf).  H query heads share KV key heads, H / KV = G each.
// The orientation of the products, the row order that feeds the accumulators of one product into the next, and the LDS images are
// those of the fused attention (attention.hip); what differs is which key blocks a query block meets (the blocks of the
// sinks, then those of the window) and, in the pass over the queries, which (query head, query block) pairs a key block meets.
//
// Rounded to bf16 on the way are P before P V and P^T dO, and dS before dS K and dS^T Q: a matrix instruction takes both operands of one type, that of v, dO, k
// and q, and fp32 ones run at a sixteenth of the rate.  Scores, maxima, sums, statistics and accumulators are fp32.  Off the definition in 64 bits by, over the values' root
// mean square: outputs 0.0021, with the derivatives 0.0024; the last rounding of results that are exact before it gives 0.0017.
#include "kernels.h"
#include "gfx950.h"
#include "head_tile.h"
#include "rows.h"

#include <utility>

namespace tbp {

// Rows at which sequence b ends.
__device__ __forceinline__ int seq_end(const int* __restrict__ lengths, int b, int S) {
  if (!lengths) return S;
  const int n = __builtin_amdgcn_readfirstlane(lengths[b]);
  return n < 0 ? 0 : n < S ? n : S;
}

// The 64-key blocks that the queries first .. last (last < n) meet: those of the sinks that lie before the window, then the window's.
struct KeyBlocks {
  int n_sink, win0, count;
  __device__ __forceinline__ KeyBlocks(int first, int last, int window, int sinks) {
    const int lo = first - window + 1;
    win0 = lo > 0 ? lo >> 6 : 0;
    const int seen_sinks = sinks < last + 1 ? sinks : last + 1;
    const int js = (seen_sinks + 63) >> 6;
    n_sink = js < win0 ? js : win0;
    count = n_sink + (last >> 6) - win0 + 1;
  }
  __device__ __forceinline__ int key0(int j) const { return (j < n_sink ? j : win0 + j - n_sink) << 6; }
};

// Sequences that lie one behind the other (PACKED): sequence b has the rows starts[b] .. starts[b + 1] - 1 of `rows`, all causal; lse and delta are [H][rows].
// The rows behind the last sequence are one without tokens, whose results are zeros.  Starts are taken as 0 .. rows and the first as 0.
// A launch has as many numbers of blocks (of queries, or of keys) as any lengths may need; those that no block has end at once.
enum { kInOrder = 1, kMostFirst };     // values of PACKED: whose block a number is
struct Packed { const int* starts; int seqs, rows; };
inline __host__ __device__ long packed_blocks(const Packed& p, int block) { return (long)p.rows / block + p.seqs + 1; }

__device__ __forceinline__ int packed_start(const Packed& p, int b) {
  const int s = b > 0 ? p.starts[b] : 0;
  return s < 0 ? 0 : s < p.rows ? s : p.rows;
}

// The sequence of a workgroup and its block in it.  n: tokens; S: rows to be written.
// LAST: query blocks, whose last ones have the most to do and come first; else key blocks, and their first ones.
struct SeqOf {
  long tok0; int n, S, block;
  // Sequence b's blocks are the numbers from starts[b] / BLOCK + b on, whose places do not overlap since a sequence has at most
  // (starts[b + 1] / BLOCK - starts[b] / BLOCK) + 1 blocks.
  template <int BLOCK, bool LAST> __device__ __forceinline__ static SeqOf in_order(const Packed& p, int number) {
    const int lane = threadIdx.x & 63;
    if (LAST) number = (int)packed_blocks(p, BLOCK) - 1 - number;
    // the last of the sequences 0 .. seqs (the rows behind them) that begins at or before this number, 64 at a time; few of them: its ends are at hand
    if (p.seqs < 63) {
      const int start = lane <= p.seqs ? packed_start(p, lane) : p.rows;
      const int b = 63 - __builtin_clzll(__ballot(lane <= p.seqs && start / BLOCK + lane <= number) | 1ull);
      const int first = __builtin_amdgcn_readlane(start, b), end = __builtin_amdgcn_readlane(start, b + 1);
      const int S = end > first ? end - first : 0;
      return SeqOf{first, b < p.seqs ? S : 0, S, number - first / BLOCK - b};
    }
    int lo = 0, size = p.seqs + 1;
    while (size > 1) {
      const int step = (size + 63) / 64, b = lo + lane * step;
      const bool before = lane * step < size && packed_start(p, b) / BLOCK + b <= number;
      const unsigned long long all = __ballot(before);               // (the first one is among them)
      const int last = all ? 63 - __builtin_clzll(all) : 0;
      lo += last * step;
      size = size - last * step < step ? size - last * step : step;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int first = packed_start(p, lo), end = lo < p.seqs ? packed_start(p, lo + 1) : p.rows;
    const int S = end > first ? end - first : 0;
    return SeqOf{first, lo < p.seqs ? S : 0, S, number - first / BLOCK - lo};
  }
  // Blocks by what they have to do, the most first, whatever sequence they are of, for up to 64 sequences, a lane each: F(j) blocks have more than j blocks of
  // their sequence from them on (of keys; of queries up to them), and those of one j go by their sequence.
  template <int BLOCK, bool LAST> __device__ __forceinline__ static SeqOf most_first(const Packed& p, int number) {
    const int lane = threadIdx.x & 63;
    const int first = lane < p.seqs ? packed_start(p, lane) : 0, end = lane < p.seqs ? packed_start(p, lane + 1) : 0;
    const int blocks = end > first ? (end - first + BLOCK - 1) / BLOCK : 0;
    int all = 0, lo = 0, step = 1, beyond = 0;     // F(lo) > number >= F(lo + 1) = beyond
    while (__any(blocks >= 64 * step)) step *= 32;         // (one look at 64 values for sequences of up to 63 blocks)
    for (bool top = true;; top = false) {          // 64 values of F at a time, a lane each
      const int j = lo + lane * step;
      int f = 0;
      for (int s = 0; s < p.seqs; s += 4)          // (lanes without a sequence have no blocks)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const int over = __builtin_amdgcn_readlane(blocks, s + i) - j;
          f += over > 0 ? over : 0;
        }
      if (top) all = __builtin_amdgcn_readfirstlane(f);
      if (number >= all) {
        const int behind = p.seqs ? packed_start(p, p.seqs) : 0;
        return SeqOf{behind, 0, p.rows - behind, number - all};
      }
      const int last = 63 - __builtin_clzll(__ballot(f > number));      // (the first one is among them; at step 1 below 63: F is 0 at the 64th)
      lo += last * step;
      beyond = __builtin_amdgcn_readlane(f, last + 1);
      if (step == 1) break;
      step /= 32;
    }
    const unsigned long long has = __ballot(blocks > lo);
    const bool mine = blocks > lo && __builtin_amdgcn_mbcnt_hi((unsigned)(has >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)has, 0)) == (unsigned)(number - beyond);
    const int who = __builtin_ctzll(__ballot(mine) | 1ull << 63);
    const int at = __builtin_amdgcn_readlane(first, who), n = __builtin_amdgcn_readlane(end, who) - at;
    return SeqOf{at, n, n, LAST ? lo : __builtin_amdgcn_readlane(blocks, who) - 1 - lo};
  }
  template <int PACKED, int BLOCK, bool LAST> __device__ __forceinline__ static SeqOf of(const Packed& p, int number) {
    return PACKED == kMostFirst ? most_first<BLOCK, LAST>(p, number) : in_order<BLOCK, LAST>(p, number);
  }
};

struct WinParams {
  const bf16_t* qkv; long ld_qkv;      // [B*S, >= (H + 2 KV) DH]: q | k | v column blocks
  bf16_t* out; long ld_out;            // [B*S, >= H*DH]
  float* lse;                          // [B, H, S]: log2 of the row's sum of exp2(score * scale * log2 e)
  const int* lengths;                  // [B] or nullptr
  Packed packed;                       // PACKED: the sequences (B 1, S rows, no window, no sinks)
  int B, H, KV, G, S, window, sinks;
  float scale_log2e;
};

// Workgroup ids run over (sequence, key head) fastest, then over the query heads of the key head, query blocks slowest: the heads
// that read the same keys then sit on one XCD (ids go round the 8 XCDs) wherever the number of key heads is a multiple of 8.
struct HeadOf {
  int b, hk, gq;                       // gq: of the key head's query heads (or groups of them)
  __device__ __forceinline__ HeadOf(int x, int B, int KV) {
    const int u = x % (B * KV);
    gq = x / (B * KV);
    b = u / KV;
    hk = u - b * KV;
  }
};

// ------------------------------------------------------------------------------------------ forward
// One workgroup = 4 waves x 32 queries of one (sequence, head); keys and values stream through LDS in blocks of 64, double-buffered,
// K one block ahead of V, the scores of the next block computed beside the exponentials of this one in a pinned order (AHEAD).
// SPLIT = 2, for grids that leave compute units idle: 64 queries per workgroup, and two waves per 32 queries, each on one 32-key tile of
// every block, whose sums meet at the end.
// No unit is full: matrix pipes are busy 54 % of the cycles that a workgroup is resident, vector instructions are issued in 56 %, and the two waves of a SIMD
// overlap them only in part, at the clock that the card's power leaves (1.8 GHz).  [2, 4096] tokens, 32 heads on 8 of 128, window 1024, 4 sinks 150 to 167 us
// over cards, 0.72 to 0.80 PFLOP/s of the pairs that are seen, 0.82 to 0.92 of those that are computed (1.14 times as many, for the tiles at the window's two
// edges).  Left out of it again: tiles of 32 keys that a wave's queries do not see, one by one (two copies of the block's code, 165 us for 152).  No more than
// the registers bounds the workgroups of a compute unit: head_dim 64, window 256, 4 sequences of 2048, 32 heads
// 49.1 us with two, 38.4 with four.
// HW: query heads of one key head that a workgroup has (PACKED), 128 / SPLIT / HW queries of each: short sequences then leave less of a block empty,
// and less of what a block computes lies behind its queries.
template <int DH, bool AHEAD, int SPLIT, int HW, int PACKED>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void window_fwd_kernel(WinParams p) {
  using HT = HeadTile<DH>;
  constexpr int KS = DH / 16, DT = DH / 32, BKV = 64, QW = 4 / SPLIT, NT = 2 / SPLIT;
  constexpr int ROWS = 128 / SPLIT, BQ = ROWS / HW;   // (query, head) rows and queries of the workgroup
  constexpr int IMG = BKV * HT::RB, SLOT = 2 * IMG;
  constexpr int NCH = IMG / 1024 / 4;                 // copies per wave per operand per block

  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  lds_u8* const lds = LDS_PTR(unsigned char, smem_raw);
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;

  const int lane = threadIdx.x & 63, ql = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int x = PACKED ? (int)blockIdx.x % (p.H / HW) : (int)blockIdx.x, y = PACKED ? (int)blockIdx.x / (p.H / HW) : (int)blockIdx.y;
  int qb = PACKED ? y : (int)gridDim.y - 1 - y;                     // last query blocks first: the first ones may have short windows
  const HeadOf at(x, p.B, p.KV);
  const int wq = SPLIT == 1 ? wave : wave % QW, wk = SPLIT == 1 ? 0 : wave / QW;      // which 32 queries, which 32-key tile of every block (SPLIT 2)
  const int b = at.b, h0 = (at.hk * (p.G / HW) + at.gq) * HW, h = h0 + wq % HW;       // the workgroup's first query head, the wave's
  SeqOf seq{(long)b * p.S, 0, p.S, qb};
  if constexpr (PACKED) { seq = SeqOf::of<PACKED, BQ, true>(p.packed, qb); qb = seq.block; }
  const int S = seq.S, window = PACKED ? 1 << 30 : p.window, sinks = PACKED ? 0 : p.sinks;
  const int q0 = qb * BQ, qw0 = q0 + 32 * (wq / HW), query = qw0 + ql;
  const long tok0 = seq.tok0, stat0 = PACKED ? (long)h * p.S + tok0 : ((long)b * p.H + h) * p.S;
  const int n = PACKED ? seq.n : seq_end(p.lengths, b, p.S);
  constexpr int LPR = DH / 8, RPI = 64 / LPR;                       // lanes per row and rows per wave-wide store
  const int rl = lane / LPR, piece = lane % LPR;

  if (q0 >= n) {                                                    // (uniform) nothing but padding
    if (wk == 0) {
      for (int r0 = 0; r0 < 32; r0 += RPI)
        if (qw0 + r0 + rl < S) *reinterpret_cast<u32x4*>(p.out + (tok0 + qw0 + r0 + rl) * p.ld_out + h * DH + 8 * piece) = u32x4{0, 0, 0, 0};
      if (g == 0 && query < S) p.lse[stat0 + query] = -INFINITY;
    }
    return;
  }
  const int q_last = (q0 + BQ < n ? q0 + BQ : n) - 1;
  const KeyBlocks kbs(q0, q_last, window, sinks);

  const typename HT::Offsets fo = HT::offsets(lane);
  // rows r0 .. of the sequence, at most `rows` of them and none from n on, as seen from column `col`
  auto rows_desc = [&](int r0, int rows, long col) {
    const int left = n - r0 < rows ? n - r0 : rows;
    return make_desc(p.qkv + (tok0 + r0) * p.ld_qkv + col, (uint32_t)((left > 0 ? left : 0) * p.ld_qkv * 2));
  };
  // ---- the block's query rows: copied (coalesced) into the second slot, which nothing else uses until they have been read
  {
    const u32x4 dq = rows_desc(q0, BQ, (long)h0 * DH);
#pragma unroll
    for (int i = 0; i < 2 * NCH / SPLIT; i++) {
      int row; unsigned go;
      HT::template plan_heads<HW>(wave + 4 * i, lane, p.ld_qkv, row, go);
      dma16(lds0 + SLOT + (wave + 4 * i) * 1024, dq, q0 + row < n ? go : kOob);
    }
  }
  int c_row[NCH];
  unsigned c_off[NCH];
#pragma unroll
  for (int i = 0; i < NCH; i++) HT::plan(wave + 4 * i, lane, p.ld_qkv, c_row[i], c_off[i]);
  const int nblk = kbs.count;
  const long kcol = (long)(p.H + at.hk) * DH, vcol = kcol + (long)p.KV * DH;
  auto issue = [&](int j, int which) {      // which: 0 the K image, 1 the V image of block j
    const int kv0 = kbs.key0(j);
    const u32x4 desc = rows_desc(kv0, BKV, which ? vcol : kcol);
    const uint32_t base = lds0 + (j & 1) * SLOT + which * IMG + wave * 1024;
#pragma unroll
    for (int i = 0; i < NCH; i++) dma16(base + i * 4096, desc, (kv0 + c_row[i] < n) ? c_off[i] : kOob);
  };

  f32x16 ot[DT];
#pragma unroll
  for (int t = 0; t < DT; t++)
#pragma unroll
    for (int e = 0; e < 16; e++) ot[t][e] = 0.f;
  // m: reference point of the row's exponentials (the same in both lane halves); l: this lane half's share of the row sum
  float m = -INFINITY, l[2] = {0.f, 0.f};

  issue(0, 0);
  issue(0, 1);
  wait_vmem<0>();
  __syncthreads();
  bf16x8 qf[KS];                       // this lane's query row as B operand of S^T = K Q^T
#pragma unroll
  for (int s = 0; s < KS; s++) qf[s] = HT::rows_frag(lds + SLOT, fo, 32 * wq, s);
  f32x16 sa[NT], sb[NT];               // S^T of the block whose softmax is in work, and of the next one
  const int wk_rows = 32 * wk * HT::RB;          // (SPLIT 2: this wave's tile of the K and V images)
  auto scores = [&](f32x16 (&st)[NT], lds_u8* kimg) {
#pragma unroll
    for (int kt = 0; kt < NT; kt++)
#pragma unroll
      for (int e = 0; e < 16; e++) st[kt][e] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; s++)
#pragma unroll
      for (int kt = 0; kt < NT; kt++)
        st[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(HT::rows_frag(kimg, fo, 32 * kt, s), qf[s], st[kt], 0, 0, 0);
  };
  if constexpr (AHEAD) {
    scores(sa, lds + wk_rows);
    __syncthreads();                   // every wave has its query row: the second slot is free
    if (nblk > 1) issue(1, 0);
  }

  auto block = [&](f32x16 (&st)[NT], f32x16 (&nx)[NT], int j) {
    wait_vmem<0>();
    __syncthreads();                   // K of block j + 1 and V of block j have landed; every wave is done with block j - 1
    if (AHEAD ? j + 2 < nblk : j + 1 < nblk) issue(AHEAD ? j + 2 : j + 1, 0);      // (not AHEAD: K of block j has landed)
    if (j + 1 < nblk) issue(j + 1, 1);
    const int kv0 = kbs.key0(j) + 32 * wk;
    if (kv0 > qw0 + 31) return;        // every key of the block is after every query of this wave
    lds_u8* const kimg = lds + ((j + 1) & 1) * SLOT + wk_rows;   // (after the last block: an older one, whose scores nobody uses)
    lds_u8* const vimg = lds + (j & 1) * SLOT + IMG + wk_rows;
    const bool low = kv0 < qw0 + 32 - window && kv0 + 32 * NT > sinks;         // some query of this wave is past the window of some key
    if (!AHEAD && low && kv0 >= sinks && kv0 + 32 * NT <= qw0 + 1 - window) return;      // ... and every query past that of every key
    bf16x8 kf[2][NT];
    if constexpr (AHEAD) {
#pragma unroll
      for (int s = 0; s < 2; s++)
#pragma unroll
        for (int kt = 0; kt < NT; kt++) kf[s][kt] = HT::rows_frag(kimg, fo, 32 * kt, s);
    } else {
      scores(st, lds + (j & 1) * SLOT + wk_rows);
    }
    if (low || kv0 + 32 * NT - 1 > qw0) {
      const int hi = query - kv0 - 4 * g, lo = hi - window, sk = sinks - kv0 - 4 * g;      // seen: <= hi, and > lo or < sk
#pragma unroll
      for (int kt = 0; kt < NT; kt++)
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int r = 32 * kt + 8 * (e >> 2) + (e & 3);
          st[kt][e] = (r > hi || (!PACKED && r <= lo && r >= sk)) ? -INFINITY : st[kt][e];
        }
    }
    // The reference point m of the exponentials has to stay within a safe distance of the running maximum, not on it: it is moved
    // (and what is accumulated rescaled) only when some query's maximum has risen by more than kSlack octaves above it.
    constexpr float kSlack = 8.f;
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < NT; kt++)
#pragma unroll
      for (int e = 0; e < 16; e++) mx = fmaxf(mx, st[kt][e]);
    mx *= p.scale_log2e;
    if (__any(mx > m + kSlack)) {
      const float mnew = fmaxf(m, fmaxf(mx, xor32(mx)));
      // (a lane that is here because of its neighbours, while its own query has seen no key yet: -inf - -inf would make NaN of its zeros)
      const float alpha = __builtin_amdgcn_exp2f(m - (mnew == -INFINITY ? 0.f : mnew));
      l[0] *= alpha;
      l[1] *= alpha;
#pragma unroll
      for (int t = 0; t < DT; t++)
#pragma unroll
        for (int e = 0; e < 16; e++) ot[t][e] *= alpha;
      m = mnew;
    }
    const float ref = m == -INFINITY ? 0.f : m;         // (no key seen yet: zeros)
    bf16x8 pb[2 * NT], vf[DT];
    auto elements = [&](int e0, int e1) {               // exponentials of elements e0 .. e1 - 1 of the lane's 16 NT
#pragma unroll
      for (int e = e0; e < e1; e++) {
        const float pe = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e >> 4][e & 15], p.scale_log2e, -ref));
        st[e >> 4][e & 15] = pe;
        l[e & 1] += pe;
        if (e % 8 == 7) pb[e >> 3] = pack8(st[e >> 4], (e >> 3) & 1);
      }
    };
    // MFMAs of the scores; elements done beside them, the rest beside all PV k-steps but the last
    constexpr int NA = NT * KS, NE = 16 * NT, EA = NT == 2 ? 18 : 10, PK = 2 * NT, PE = PK - 1;
    static_assert(EA >= 8 && EA + (NE - EA) / PE >= 16 && (NT == 1 || EA + (NE - EA) * 2 / PE >= 24), "P must be ready in time");
    if constexpr (AHEAD) {
#pragma unroll
      for (int kt = 0; kt < NT; kt++)
#pragma unroll
        for (int e = 0; e < 16; e++) nx[kt][e] = 0.f;
    }
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (AHEAD) {
#pragma unroll
      for (int i = 0; i < NA; i++) {
        const int s = i / NT, kt = i % NT;
        nx[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s & 1][kt], qf[s], nx[kt], 0, 0, 0);
        if (s + 2 < KS) kf[s & 1][kt] = HT::rows_frag(kimg, fo, 32 * kt, s + 2);
        if (i >= NA - DT) vf[i - (NA - DT)] = HT::cols_frag(vimg, fo, 0, 0, i - (NA - DT));
        elements(EA * i / NA, EA * (i + 1) / NA);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int t = 0; t < DT; t++) vf[t] = HT::cols_frag(vimg, fo, 0, 0, t);
      elements(0, EA);
    }
#pragma unroll
    for (int i = 0; i < PK * DT; i++) {
      const int ku = i / DT, t = i % DT;
      ot[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[t], pb[ku], ot[t], 0, 0, 0);
      if (ku < PE) vf[t] = HT::cols_frag(vimg, fo, 32 * ((ku + 1) >> 1), (ku + 1) & 1, t);
      if (ku < PE) elements(EA + (NE - EA) * i / (PE * DT), EA + (NE - EA) * (i + 1) / (PE * DT));
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };
  for (int j = 0; j < nblk; j += 2) {
    block(sa, sb, j);
    if (j + 1 < nblk) block(sb, sa, j + 1);
  }

  // ---- o = O^T / l, transposed back through LDS (rows padded against bank conflicts) and written as whole rows
  __syncthreads();
  constexpr int EROW = DH * 2 + 16;
  static_assert(ROWS * EROW <= 2 * SLOT, "the output tile must fit in the ring");
  lds_u8* const erow = lds + 32 * wq * EROW;
  float lq = (l[0] + l[1]) + xor32(l[0] + l[1]);
  if constexpr (SPLIT == 2) {
    // the two waves of a query: what the second one summed, brought to the common reference point, joins the first one's
    static_assert(ROWS * EROW + 1024 <= SLOT && QW * DT * 4096 <= SLOT, "output tile, statistics and partial sums side by side");
    LDS_AS float* const part = reinterpret_cast<LDS_AS float*>(lds + SLOT) + wq * (DT * 1024);
    LDS_AS float* const stat = reinterpret_cast<LDS_AS float*>(lds + ROWS * EROW) + wq * 128;
    if (wk == 1) {
#pragma unroll
      for (int t = 0; t < DT; t++)
#pragma unroll
        for (int e = 0; e < 16; e++) part[(t * 16 + e) * 64 + lane] = ot[t][e];
      stat[lane] = m;
      stat[64 + lane] = lq;
    }
    __syncthreads();
    if (wk == 1) return;
    const float m1 = stat[lane], mc = fmaxf(m, m1);
    const float f0 = __builtin_amdgcn_exp2f(m - mc), f1 = __builtin_amdgcn_exp2f(m1 - mc);
    m = mc;
    lq = lq * f0 + stat[64 + lane] * f1;
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
      for (int e = 0; e < 16; e++) ot[t][e] = ot[t][e] * f0 + part[(t * 16 + e) * 64 + lane] * f1;
  }
  {
    const bool live = PACKED || query < n;              // (padding: zeros, whatever the lane holds)
    const float inv = 1.f / lq;
#pragma unroll
    for (int t = 0; t < DT; t++)
#pragma unroll
      for (int e4 = 0; e4 < 4; e4++) {
        bf16x4 v;
#pragma unroll
        for (int r = 0; r < 4; r++) v[r] = (bf16_t)(live ? ot[t][4 * e4 + r] * inv : 0.f);
        *reinterpret_cast<LDS_AS bf16x4*>(erow + ql * EROW + (32 * t + 8 * e4 + 4 * g) * 2) = v;
      }
    if (g == 0 && query < S) p.lse[stat0 + query] = live ? m + __builtin_amdgcn_logf(lq) : -INFINITY;
  }
  // (LDS operations of a wave execute in order: the reads below see this wave's own writes above)
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += RPI) {
    const int qrow = qw0 + r0 + rl;
    if (qrow < S)
      *reinterpret_cast<u32x4*>(p.out + (tok0 + qrow) * p.ld_out + h * DH + 8 * piece) =
          *reinterpret_cast<const LDS_AS u32x4*>(erow + (r0 + rl) * EROW + 16 * piece);
  }
}

// ------------------------------------------------------------------------------------------ backward-p1: dQ and delta
// dQ = scale * dS K: oriented like the forward, per 32-key tile S^T and dP^T = V dO^T are rebuilt, dS^T = P^T (dP^T - delta) is fed into
// dQ^T += K^T dS^T.  delta = rowsum(dout * out) of its queries is computed first and left for the pass over the queries.
// One workgroup = 4 waves x 32 queries, key blocks through LDS in two slots, as in the forward, so that the sum over the keys stays in registers and
// no atomics are needed.  As in the forward no unit is full, at the clock that the power leaves: 8192 tokens, 32 heads on 8 of 128, window 2048, 4 sinks 355 to 378
// us, 0.96 to 1.02 PFLOP/s of the three products over the seen pairs, matrix pipes busy 56 %, vector instructions 45 %.
struct WinDqParams {
  const bf16_t* qkv; long ld_qkv;
  const bf16_t* dout; const bf16_t* out; long ld_do;
  const float* lse;                    // [B, H, S]
  float* delta;                        // [B, H, S]: written here for the tokens that are there
  const int* lengths;
  Packed packed;
  bf16_t* dqkv; long ld_dqkv;
  int B, H, KV, G, S, window, sinks;
  float scale, scale_log2e;
};

template <int DH, int SPLIT, int HW, int PACKED>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void window_bwd_dq_kernel(WinDqParams p) {
  using HT = HeadTile<DH>;
  constexpr int KS = DH / 16, DT = DH / 32, BKV = 64, QW = 4 / SPLIT;
  constexpr int ROWS = 128 / SPLIT, BQ = ROWS / HW;
  constexpr int IMG = BKV * HT::RB, SLOT = 2 * IMG;
  constexpr int NCH = IMG / 1024 / 4;

  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  lds_u8* const lds = LDS_PTR(unsigned char, smem_raw);
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;

  const int lane = threadIdx.x & 63, ql = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int x = PACKED ? (int)blockIdx.x % (p.H / HW) : (int)blockIdx.x, y = PACKED ? (int)blockIdx.x / (p.H / HW) : (int)blockIdx.y;
  int qb = PACKED ? y : (int)gridDim.y - 1 - y;
  const HeadOf at(x, p.B, p.KV);
  const int wq = SPLIT == 1 ? wave : wave % QW, wk = SPLIT == 1 ? 0 : wave / QW;      // which 32 queries, which 32-key tile of every block (SPLIT 2)
  const int b = at.b, h0 = (at.hk * (p.G / HW) + at.gq) * HW, h = h0 + wq % HW;       // the workgroup's first query head, the wave's
  SeqOf seq{(long)b * p.S, 0, p.S, qb};
  if constexpr (PACKED) { seq = SeqOf::of<PACKED, BQ, true>(p.packed, qb); qb = seq.block; }
  const int S = seq.S, window = PACKED ? 1 << 30 : p.window, sinks = PACKED ? 0 : p.sinks;
  const int q0 = qb * BQ, qw0 = q0 + 32 * (wq / HW), query = qw0 + ql;
  const long tok0 = seq.tok0, stat0 = PACKED ? (long)h * p.S + tok0 : ((long)b * p.H + h) * p.S;
  const int n = PACKED ? seq.n : seq_end(p.lengths, b, p.S);
  constexpr int LPR = DH / 8, RPI = 64 / LPR;
  const int rl = lane / LPR, piece = lane % LPR;

  if (q0 >= n) {
    if (wk == 0)
      for (int r0 = 0; r0 < 32; r0 += RPI)
        if (qw0 + r0 + rl < S) *reinterpret_cast<u32x4*>(p.dqkv + (tok0 + qw0 + r0 + rl) * p.ld_dqkv + h * DH + 8 * piece) = u32x4{0, 0, 0, 0};
    return;
  }
  const int q_last = (q0 + BQ < n ? q0 + BQ : n) - 1;
  const KeyBlocks kbs(q0, q_last, window, sinks);

  const typename HT::Offsets fo = HT::offsets(lane);
  auto rows_desc = [&](const bf16_t* base, long ld, int r0, int rows, long col) {
    const int left = n - r0 < rows ? n - r0 : rows;
    return make_desc(base + (tok0 + r0) * ld + col, (uint32_t)((left > 0 ? left : 0) * ld * 2));
  };
  // ---- the block's query rows into the second slot and their output derivatives into the first (coalesced copies)
  {
    const u32x4 dq = rows_desc(p.qkv, p.ld_qkv, q0, BQ, (long)h0 * DH), dd = rows_desc(p.dout, p.ld_do, q0, BQ, (long)h0 * DH);
#pragma unroll
    for (int i = 0; i < 2 * NCH / SPLIT; i++) {
      int row; unsigned go, gd;
      HT::template plan_heads<HW>(wave + 4 * i, lane, p.ld_qkv, row, go);
      HT::template plan_heads<HW>(wave + 4 * i, lane, p.ld_do, row, gd);
      const bool ok = q0 + row < n;
      dma16(lds0 + SLOT + (wave + 4 * i) * 1024, dq, ok ? go : kOob);
      dma16(lds0 + (wave + 4 * i) * 1024, dd, ok ? gd : kOob);
    }
  }
  int c_row[NCH];
  unsigned c_off[NCH];
#pragma unroll
  for (int i = 0; i < NCH; i++) HT::plan(wave + 4 * i, lane, p.ld_qkv, c_row[i], c_off[i]);
  const int nblk = kbs.count;
  const long kcol = (long)(p.H + at.hk) * DH, vcol = kcol + (long)p.KV * DH;
  auto issue = [&](int j) {
    const int kv0 = kbs.key0(j);
    const u32x4 dk = rows_desc(p.qkv, p.ld_qkv, kv0, BKV, kcol), dv = rows_desc(p.qkv, p.ld_qkv, kv0, BKV, vcol);
    const uint32_t base = lds0 + (j & 1) * SLOT + wave * 1024;
#pragma unroll
    for (int i = 0; i < NCH; i++) {
      const unsigned off = (kv0 + c_row[i] < n) ? c_off[i] : kOob;
      dma16(base + i * 4096, dk, off);
      dma16(base + IMG + i * 4096, dv, off);
    }
  };
  const bool qlive = query < n;
  const float lse_q = qlive ? p.lse[stat0 + query] : 0.f;

  f32x16 dqt[DT];
#pragma unroll
  for (int t = 0; t < DT; t++)
#pragma unroll
    for (int e = 0; e < 16; e++) dqt[t][e] = 0.f;

  wait_vmem<0>();
  __syncthreads();
  bf16x8 qf[KS], dof[KS];            // this lane's query row and output-derivative row as B operands
#pragma unroll
  for (int s = 0; s < KS; s++) {
    qf[s] = HT::rows_frag(lds + SLOT, fo, 32 * wq, s);
    dof[s] = HT::rows_frag(lds, fo, 32 * wq, s);
  }
  __syncthreads();                   // every wave has its rows: both slots are free for the key blocks
  issue(0);
  // ---- delta: the block's rows of the output arrive in the second slot beside the first key block
  {
    const u32x4 dr = rows_desc(p.out, p.ld_do, q0, BQ, (long)h0 * DH);
#pragma unroll
    for (int i = 0; i < 2 * NCH / SPLIT; i++) {
      int row; unsigned go;
      HT::template plan_heads<HW>(wave + 4 * i, lane, p.ld_do, row, go);
      dma16(lds0 + SLOT + (wave + 4 * i) * 1024, dr, q0 + row < n ? go : kOob);
    }
  }
  wait_vmem<0>();
  __syncthreads();
  float dl_q = 0.f;
#pragma unroll
  for (int s = 0; s < KS; s++) {
    const bf16x8 o = HT::rows_frag(lds + SLOT, fo, 32 * wq, s);
#pragma unroll
    for (int i = 0; i < 8; i++) dl_q += (float)o[i] * (float)dof[s][i];
  }
  dl_q += xor32(dl_q);
  if (qlive && g == 0 && wk == 0) p.delta[stat0 + query] = dl_q;
  __syncthreads();                   // the second slot is free again
  for (int j = 0; j < nblk; j++) {
    wait_vmem<0>();
    __syncthreads();                 // block j has landed; every wave is done with the other slot
    if (j + 1 < nblk) issue(j + 1);
    const int kv0 = kbs.key0(j);
    lds_u8* const kimg = lds + (j & 1) * SLOT;
    lds_u8* const vimg = kimg + IMG;
    const int hi = query - kv0 - 4 * g, lo = hi - window, sk = sinks - kv0 - 4 * g;      // seen: <= hi, and > lo or < sk
#pragma unroll 1
    for (int kt = SPLIT == 2 ? wk : 0; kt < (SPLIT == 2 ? wk + 1 : 2); kt++) {
      const int t0 = kv0 + 32 * kt;  // (uniform over the wave) tiles that none of its queries sees a key of
      if (t0 > qw0 + 31 || (t0 >= sinks && t0 + 32 <= qw0 + 1 - window)) continue;
      const bool edge = t0 + 31 > qw0 || (t0 < qw0 + 32 - window && t0 + 32 > sinks);
      f32x16 st, dp;
#pragma unroll
      for (int e = 0; e < 16; e++) { st[e] = 0.f; dp[e] = 0.f; }
      // (the order is pinned: the compiler would fetch each fragment right before its MFMA)
      constexpr int PF = 3;
      bf16x8 kf[PF], vf[PF], ktf[DT];
#pragma unroll
      for (int s = 0; s < PF; s++) { kf[s] = HT::rows_frag(kimg, fo, 32 * kt, s); vf[s] = HT::rows_frag(vimg, fo, 32 * kt, s); }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < KS; s++) {
        st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s % PF], qf[s], st, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[s % PF], dof[s], dp, 0, 0, 0);
        if (s + PF < KS) { kf[s % PF] = HT::rows_frag(kimg, fo, 32 * kt, s + PF); vf[s % PF] = HT::rows_frag(vimg, fo, 32 * kt, s + PF); }
        if (s >= KS - DT) ktf[s - (KS - DT)] = HT::cols_frag(kimg, fo, 32 * kt, 0, s - (KS - DT));
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int e = 0; e < 16; e++) st[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], p.scale_log2e, -lse_q));
      if (edge) {
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int r = 32 * kt + 8 * (e >> 2) + (e & 3);
          st[e] = (r > hi || (!PACKED && r <= lo && r >= sk)) ? 0.f : st[e];
        }
      }
#pragma unroll
      for (int e = 0; e < 16; e++) st[e] *= dp[e] - dl_q;    // dS^T
#pragma unroll
      for (int u = 0; u < 2; u++) {
        const bf16x8 sb = pack8(st, u);
#pragma unroll
        for (int t = 0; t < DT; t++) {
          dqt[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ktf[t], sb, dqt[t], 0, 0, 0);
          if (u == 0) ktf[t] = HT::cols_frag(kimg, fo, 32 * kt, 1, t);     // the second k-step's fragment, behind the MFMA that used the first
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }

  __syncthreads();
  if constexpr (SPLIT == 2) {        // the two waves of a query add up, first the wave of the first tiles
    LDS_AS float* const part = reinterpret_cast<LDS_AS float*>(lds) + wq * (DT * 1024);
    static_assert(QW * DT * 4096 <= 2 * SLOT, "the partial sums must fit in the ring");
    if (wk == 1) {
#pragma unroll
      for (int t = 0; t < DT; t++)
#pragma unroll
        for (int e = 0; e < 16; e++) part[(t * 16 + e) * 64 + lane] = dqt[t][e];
    }
    __syncthreads();
    if (wk == 0) {
#pragma unroll
      for (int t = 0; t < DT; t++)
#pragma unroll
        for (int e = 0; e < 16; e++) dqt[t][e] += part[(t * 16 + e) * 64 + lane];
    }
    __syncthreads();
    if (wk == 1) return;
  }
  constexpr int EROW = DH * 2 + 16;
  static_assert(ROWS * EROW <= 2 * SLOT, "the output tile must fit in the ring");
  lds_u8* const erow = lds + 32 * wq * EROW;
#pragma unroll
  for (int t = 0; t < DT; t++)
#pragma unroll
    for (int e4 = 0; e4 < 4; e4++) {
      bf16x4 v;
#pragma unroll
      for (int r = 0; r < 4; r++) v[r] = (bf16_t)(PACKED || qlive ? dqt[t][4 * e4 + r] * p.scale : 0.f);
      *reinterpret_cast<LDS_AS bf16x4*>(erow + ql * EROW + (32 * t + 8 * e4 + 4 * g) * 2) = v;
    }
  // (LDS operations of a wave execute in order: the reads below see this wave's own writes above)
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += RPI) {
    const int qrow = qw0 + r0 + rl;
    if (qrow < S)
      *reinterpret_cast<u32x4*>(p.dqkv + (tok0 + qrow) * p.ld_dqkv + h * DH + 8 * piece) =
          *reinterpret_cast<const LDS_AS u32x4*>(erow + (r0 + rl) * EROW + 16 * piece);
  }
}

// ------------------------------------------------------------------------------------------ backward-p1: dK and dV
// One workgroup = 128 keys (64: see window_parts) of one (sequence, key head) and a part of the (query head of the group, 64-query step) pairs that see them,
// walked as one list, so that dK and dV of shared heads add up in the accumulators.  The key blocks of the sinks are seen by every
// later query, not just by a window of them: their lists are longer, and cut into parts of about the length of the
// others'.  Lists are also cut where the key blocks alone are too few to fill the chip.  A key block of one part is written as it is;
// the parts of others leave fp32 partial sums that a second launch adds up in order.
// Roles of the waves as in the fused attention's pass: 4 "left" waves compute P and dS of their 32 keys and hand them over through
// LDS, 4 "right" waves issue all copies and accumulate dV^T += dO^T P, dK^T += Q^T dS of one 32-query tile later.
// 8192 tokens, 32 heads on 8 of 128, window 2048, 4 sinks 535 to 570 us, 0.85 to 0.90 PFLOP/s of the four products over the seen pairs, at the clock that the power
// leaves: matrix pipes busy 50 %, the LDS 44 %, vector instructions 29 %; a step of the left waves and one of the right waves meet at every barrier.  Of the tiles
// that the right waves multiply 4 % are zeros because no pair of them is seen (window 2048; 128 with 64 keys 17 %).  Short windows are bound by the chain of a step (scores,
// exponentials, hand-over, barrier) in few workgroups: 12 heads on 4 of 64, 4 ragged sequences of 1001, window 300 19 us.  Tried at head_dim 128: lse and delta
// fetched by the left waves, 20 us more; with 64 keys, and the LDS so freed a fourth slot, copies a step earlier: 177 -> 184 us at 2 of 4096, window 128.
struct WinKvParams {
  const bf16_t* qkv; long ld_qkv;
  const bf16_t* dout; long ld_do;
  const float* lse;
  const float* delta;
  const int* lengths;
  Packed packed;
  bf16_t* dqkv; long ld_dqkv;
  float* partial;                      // [B KV][sum of parts over the key blocks that are cut][2][KEYS][DH]
  int B, H, KV, G, S, window, sinks;
  WindowParts parts;
  float scale, scale_log2e;
};

// Lane I of every 16 lanes' own row, to all of the row.
template <int I> __device__ __forceinline__ float row_lane(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x150 + I, 0xf, 0xf, true));
}
template <typename F, int... I> __device__ __forceinline__ void each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

template <int DH, int KEYS, int PACKED>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(DH == 64 ? 4 : 2))) void window_bwd_kv_kernel(WinKvParams p) {
  using HT = HeadTile<DH>;
  constexpr int KS = DH / 16, DT = DH / 32, BQ = 64;
  constexpr int KB = KEYS / 32, TPI = 4 / KB;                 // 32-key blocks of the workgroup; 32-query tiles per iteration
  constexpr bool OWN = DH == 64;                              // the left waves fetch lse and delta themselves
  constexpr int IMG = BQ * HT::RB, SLOT = 2 * IMG + (OWN ? 0 : 1024);      // Q image, dO image, 64 x (lse, delta) unless OWN; three slots
  constexpr int NCH = IMG / 1024 / 4;                         // copies per right wave and image
  constexpr int OPS = 2 * NCH + !OWN;                           // vector-memory operations of one issue(), per right wave
  constexpr int HAND = 4 * 4096;                              // one hand-over buffer: 4 wave pairs x 64 lanes x 64 bytes
  constexpr int HALF = 32 * HT::RB;                           // the second tile's rows inside an image

  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  lds_u8* const lds = LDS_PTR(unsigned char, smem_raw);
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  lds_u8* const hand = lds + 3 * SLOT;

  const int tid = threadIdx.x, lane = tid & 63, kl = lane & 31, g = lane >> 5;
  const int wave8 = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int right = wave8 >> 2, wave = wave8 & 3;             // role
  const int kblk = KB == 4 ? wave : wave % KB, tq_left = KB == 4 ? 0 : wave / KB;      // a left wave's 32 keys of the block, and its tile of an iteration
  const int b = PACKED ? 0 : (int)blockIdx.x / p.KV, hk = (int)blockIdx.x % p.KV;
  const int y = PACKED ? (int)blockIdx.x / p.KV : (int)blockIdx.y;
  const bool sink_block = !PACKED && y < p.parts.sink_blocks * p.parts.sink_parts;
  const int np = sink_block ? p.parts.sink_parts : p.parts.other_parts;
  const int yy = sink_block ? y : y - (PACKED ? 0 : p.parts.sink_blocks * p.parts.sink_parts);
  const int number = yy / np + (PACKED || sink_block ? 0 : p.parts.sink_blocks), part = yy % np;
  SeqOf seq{(long)b * p.S, 0, p.S, number};
  if constexpr (PACKED) seq = SeqOf::of<PACKED, KEYS, false>(p.packed, number);
  const int kb = seq.block, S = seq.S, window = PACKED ? 1 << 30 : p.window, sinks = PACKED ? 0 : p.sinks;
  const int kv0 = kb * KEYS, kw0 = kv0 + 32 * kblk, key = kw0 + kl;
  const long tok0 = seq.tok0;
  const int n = PACKED ? seq.n : seq_end(p.lengths, b, p.S);
  if (PACKED && kv0 >= S) return;                             // (uniform) a number that no block has
  // lse and delta of query head h's rows of the sequence
  auto stat0 = [&](int h) { return PACKED ? (long)h * p.S + tok0 : ((long)b * p.H + h) * p.S; };
  const typename HT::Offsets fo = HT::offsets(lane);
  // steps of 64 queries that see the block, for each of the G query heads; this part's share of the G * nst pairs
  const int step0 = kv0 / BQ, nq = (n + BQ - 1) / BQ;
  int step1 = nq;
  if (kv0 >= sinks && (long)kv0 + KEYS + window - 2 < n) step1 = (kv0 + KEYS + window - 2) / BQ + 1;
  const int nst = step1 > step0 ? step1 - step0 : 0;
  const int total = p.G * nst, share = (total + np - 1) / np;
  const int i0 = part * share < total ? part * share : total, i1 = i0 + share < total ? i0 + share : total;
  const int nt = 2 * (i1 - i0) / TPI;                         // iterations
  const int hq0 = nst ? i0 / nst : 0, sq0 = nst ? step0 + i0 - hq0 * nst : 0;      // the first pair
  typedef LDS_AS float lds_f32;
  lds_u8* const my_hand = hand + wave * 4096 + lane * 16;     // + buffer * HAND + 1024 * {p0, p1, s0, s1}
  constexpr int KVIMG = KEYS * HT::RB;                        // image of the block's K (then V) rows
  lds_u8* const kvimg = lds + 2 * SLOT;
  static_assert(2 * KVIMG <= SLOT + 2 * HAND, "K and V images must fit in the third slot plus the hand-over area");
  // 32 x 32 tiles of queries from q and keys from k of which no pair is seen; and of which every pair is
  auto unseen = [&](int q, int k) { return q + 31 < k || (q - (k + 31) >= window && k >= sinks); };
  auto whole = [&](int q, int k) { return q >= k + 31 && (q + 31 - k < window || k + 32 <= sinks); };

  if (!right) {
    // ------------------------------------------------------------------ left: S, dP, P, dS
    bf16x8 kfb[KS], vfb[KS];
    __syncthreads();                                          // the first two steps and the K / V rows have landed
#pragma unroll
    for (int s = 0; s < KS; s++) {
      kfb[s] = HT::rows_frag(kvimg, fo, 32 * kblk, s);
      vfb[s] = HT::rows_frag(kvimg + KVIMG, fo, 32 * kblk, s);
    }
    __syncthreads();                                          // every left wave has its rows: the area is free again
    int st_at = sq0;                                          // the step that tile `it` lies in
    // (OWN) lse and delta of the tile's queries, fetched an iteration ahead: lane i of 16 keeps those of register i of its half (below).
    // Without room for them in the LDS two workgroups fit a compute unit.
    static_assert(!OWN || TPI == 2, "a step per iteration");
    const int sq = 8 * ((lane & 15) >> 2) + 4 * g + (lane & 3) + 32 * tq_left;
    float next_ls = 0.f, next_dl = 0.f;
    int sl_i = i0, sl_h = hq0, sl_st = sq0;
    auto fetch_stats = [&] {
      const int q = sl_st * BQ + sq;
      const long at = stat0(hk * p.G + sl_h) + q;
      next_ls = next_dl = 0.f;                                // (rows past the end: zeros, which with zero rows of Q and dO add nothing)
      if (sl_i < i1 && q < n) { next_ls = p.lse[at]; next_dl = p.delta[at]; }
      sl_i++;
      if (++sl_st == step1) { sl_st = step0; sl_h++; }
    };
    if constexpr (OWN) fetch_stats();
    const int past = key >= sinks ? key + window : 0x7fffffff;      // the first query past the lane's key's window
    for (int it = 0; it <= nt; it++) {
      const int tile = TPI * it + tq_left, qt0 = st_at * BQ + 32 * (tile & 1);
      lds_u8* const out = my_hand + (it & 1) * HAND;
      const float my_ls = next_ls, my_dl = next_dl;
      if constexpr (OWN) fetch_stats();
      if (it < nt && unseen(qt0, kw0)) {
#pragma unroll
        for (int i = 0; i < 4; i++) *reinterpret_cast<LDS_AS u32x4*>(out + 1024 * i) = u32x4{0, 0, 0, 0};
      } else if (it < nt) {
        lds_u8* const slot = lds + ((tile >> 1) % 3) * SLOT;
        lds_u8* const qimg = slot + (tile & 1) * HALF;
        lds_u8* const dimg = qimg + IMG;
        const lds_f32* const stat = reinterpret_cast<const lds_f32*>(slot + 2 * IMG) + 32 * (tile & 1);
        f32x16 sa, da;
#pragma unroll
        for (int e = 0; e < 16; e++) { sa[e] = 0.f; da[e] = 0.f; }
        constexpr int PF = KS < 4 ? KS : 4;
        bf16x8 fq[KS], fd[KS];
        f32x4 ls[4], dl[4];
#pragma unroll
        for (int s = 0; s < PF; s++) { fq[s] = HT::rows_frag(qimg, fo, 0, s); fd[s] = HT::rows_frag(dimg, fo, 0, s); }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < KS; s++) {
          if (s + PF < KS) { fq[s + PF] = HT::rows_frag(qimg, fo, 0, s + PF); fd[s + PF] = HT::rows_frag(dimg, fo, 0, s + PF); }
          if (!OWN && s >= KS - 4) {
            const int e4 = s - (KS - 4);
            ls[e4] = *reinterpret_cast<const LDS_AS f32x4*>(stat + 8 * e4 + 4 * g);
            dl[e4] = *reinterpret_cast<const LDS_AS f32x4*>(stat + BQ + 8 * e4 + 4 * g);
          }
          sa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[s], kfb[s], sa, 0, 0, 0);
          da = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fd[s], vfb[s], da, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        // register e of the tile is query qt0 + 8 (e / 4) + 4 g + e % 4
        float pv[16], sv[16];
        if constexpr (OWN)
          each([&](auto i) { ls[i >> 2][i & 3] = row_lane<i>(my_ls); dl[i >> 2][i & 3] = row_lane<i>(my_dl); }, std::make_integer_sequence<int, 16>());
#pragma unroll
        for (int e = 0; e < 16; e++) pv[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sa[e], p.scale_log2e, -ls[e >> 2][e & 3]));
        if (!whole(qt0, kw0)) {
          const int lo = key - qt0 - 4 * g, hi = past - qt0 - 4 * g;
#pragma unroll
          for (int e = 0; e < 16; e++) {
            const int r = 8 * (e >> 2) + (e & 3);
            pv[e] = (r < lo || (!PACKED && r >= hi)) ? 0.f : pv[e];
          }
        }
#pragma unroll
        for (int e = 0; e < 16; e++) sv[e] = pv[e] * (da[e] - dl[e >> 2][e & 3]);
        bf16x8 kp[2], ks[2];
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
          for (int t = 0; t < 8; t++) { kp[u][t] = (bf16_t)pv[8 * u + t]; ks[u][t] = (bf16_t)sv[8 * u + t]; }
        *reinterpret_cast<LDS_AS bf16x8*>(out) = kp[0];
        *reinterpret_cast<LDS_AS bf16x8*>(out + 1024) = kp[1];
        *reinterpret_cast<LDS_AS bf16x8*>(out + 2048) = ks[0];
        *reinterpret_cast<LDS_AS bf16x8*>(out + 3072) = ks[1];
      }
      if (TPI == 2 || (it & 1)) st_at = st_at + 1 == step1 ? step0 : st_at + 1;
      __syncthreads();
    }
    __syncthreads();                                          // every right wave's copies have landed: the ring is free
    __syncthreads();                                          // the right waves have put dK and dV into LDS (below)
    return;
  }

  // -------------------------------------------------------------------- right: copies, dV^T, dK^T
  int c_row[NCH];
  unsigned cq_off[NCH], cd_off[NCH];
#pragma unroll
  for (int i = 0; i < NCH; i++) {
    HT::plan(wave + 4 * i, lane, p.ld_qkv, c_row[i], cq_off[i]);
    HT::plan(wave + 4 * i, lane, p.ld_do, c_row[i], cd_off[i]);
  }
  // Called once for every pair in order.  Every call issues exactly OPS operations per wave (pairs past the end write zeros into their
  // slot and fetch nothing), so a wait for "all but the last issue" is a fixed count.
  int is_i = i0, is_h = hq0, is_st = sq0;
  auto issue = [&] {
    const bool live = is_i < i1;
    const int q0 = live ? is_st * BQ : 0, h = hk * p.G + (live ? is_h : 0);
    const uint32_t slot = lds0 + ((is_i - i0) % 3) * SLOT;
    const int left = live ? (n - q0 < BQ ? n - q0 : BQ) : 0;
    const u32x4 dq = make_desc(p.qkv + (tok0 + q0) * p.ld_qkv + (long)h * DH, (uint32_t)(left * p.ld_qkv * 2));
    const u32x4 dd = make_desc(p.dout + (tok0 + q0) * p.ld_do + (long)h * DH, (uint32_t)(left * p.ld_do * 2));
#pragma unroll
    for (int c = 0; c < NCH; c++) {
      const bool ok = c_row[c] < left;
      dma16(slot + wave * 1024 + c * 4096, dq, ok ? cq_off[c] : kOob);
      dma16(slot + IMG + wave * 1024 + c * 4096, dd, ok ? cd_off[c] : kOob);
    }
    if constexpr (!OWN) {
      // row statistics: wave 0 fetches lse[0..63], wave 1 delta[0..63]; waves 2 and 3 issue the same instruction out of range (nothing
      // moves) to keep the count uniform.  (Rows past the end: zeros, as above.)
      const u32x4 ds = make_desc(((wave & 1) == 0 ? p.lse : p.delta) + stat0(h) + q0, (uint32_t)(left * 4));
      dma4(slot + 2 * IMG + wave * 256, ds, wave < 2 && lane < left ? (unsigned)(lane * 4) : kOob);
    }
    is_i++;
    if (++is_st == step1) { is_st = step0; is_h++; }
  };
  // A right wave owns 32 head-dim columns (its index) of dV^T and dK^T for all four key blocks of the workgroup.  With head_dim 64 waves
  // 2 and 3 have no columns and only copy.
  f32x16 dvt[KB], dkt[KB];
#pragma unroll
  for (int t = 0; t < KB; t++)
#pragma unroll
    for (int e = 0; e < 16; e++) { dvt[t][e] = 0.f; dkt[t][e] = 0.f; }
  const bool has_cols = wave < DT;
  int col0 = 0, col1 = 0;                                     // fragment offsets of this wave's column block
#pragma unroll
  for (int t = 0; t < DT; t++)
    if (t == wave) { col0 = fo.cols[t][0]; col1 = fo.cols[t][1]; }
  auto my_cols = [&](lds_u8* img, int u) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_AS s16x4*>(img + col0 + 16 * u * HT::RB));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LDS_AS s16x4*>(img + col1 + 16 * u * HT::RB));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  {  // the block's K and V rows, for the left waves
    const int left = n - kv0 < KEYS ? n - kv0 : KEYS;         // (may be negative: no rows)
    const bf16_t* kb0 = p.qkv + (tok0 + kv0) * p.ld_qkv + (long)(p.H + hk) * DH;
    const uint32_t bytes = (uint32_t)((left > 0 ? left : 0) * p.ld_qkv * 2);
    const u32x4 dk = make_desc(kb0, bytes), dv = make_desc(kb0 + (long)p.KV * DH, bytes);
#pragma unroll
    for (int i = 0; i < NCH * KEYS / 64; i++) {
      int row; unsigned go;
      HT::plan(wave + 4 * i, lane, p.ld_qkv, row, go);
      const unsigned off = row < left ? go : kOob;
      dma16(lds0 + 2 * SLOT + (wave + 4 * i) * 1024, dk, off);
      dma16(lds0 + 2 * SLOT + KVIMG + (wave + 4 * i) * 1024, dv, off);
    }
  }
  issue();
  issue();
  wait_vmem<0>();
  __syncthreads();
  __syncthreads();                                            // the left waves have read their K and V rows
  for (int it = 0; it <= nt; it++) {
    if (it > 0 && has_cols) {
#pragma unroll
      for (int tq = 0; tq < TPI; tq++) {
        const int tile = TPI * (it - 1) + tq;
        lds_u8* const qimg = lds + ((tile >> 1) % 3) * SLOT + (tile & 1) * HALF;
        lds_u8* const dimg = qimg + IMG;
        // this wave's 32 head-dim columns of dO^T and Q^T (two k-steps of 16 queries), then every key block's P and dS, each
        // fetched one key block ahead of its MFMAs (pinned, as on the left)
        bf16x8 fo_d[2], fo_q[2], kp[2][2], ks[2][2];
        const lds_u8* const in = hand + ((it - 1) & 1) * HAND + tq * (KB * 4096) + lane * 16;
        auto fetch = [&](int kbk) {
#pragma unroll
          for (int u = 0; u < 2; u++) {
            kp[kbk & 1][u] = *reinterpret_cast<const LDS_AS bf16x8*>(in + kbk * 4096 + 1024 * u);
            ks[kbk & 1][u] = *reinterpret_cast<const LDS_AS bf16x8*>(in + kbk * 4096 + 2048 + 1024 * u);
          }
        };
#pragma unroll
        for (int u = 0; u < 2; u++) { fo_d[u] = my_cols(dimg, u); fo_q[u] = my_cols(qimg, u); }
        fetch(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kbk = 0; kbk < KB; kbk++) {
          if (kbk + 1 < KB) fetch(kbk + 1);
#pragma unroll
          for (int u = 0; u < 2; u++) {
            dvt[kbk] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fo_d[u], kp[kbk & 1][u], dvt[kbk], 0, 0, 0);
            dkt[kbk] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fo_q[u], ks[kbk & 1][u], dkt[kbk], 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    if constexpr (TPI == 1) {
      // Pair (it + 1) / 2 is what the left waves start at the next iteration, when `it` is odd: it was issued three barriers ago and only
      // the issue after it may still be in flight
      if (it & 1) wait_vmem<OPS>();
      __syncthreads();
      // after this barrier nobody reads the pair before it / 2 any more (it even): its slot takes pair it / 2 + 2
      if (!(it & 1)) issue();
    } else {
      // a whole pair per iteration: the one after the left waves' was issued behind the barrier before, and the one before it, which the
      // right waves have just finished, leaves its slot to the pair after next
      wait_vmem<0>();
      __syncthreads();
      issue();
    }
  }
  wait_vmem<0>();                                             // (copies past the end: zeros, no traffic)
  __syncthreads();                                            // ... of every wave, before the ring is reused below

  if (np > 1) {
    // a part of the sums, dK unscaled: [2][KEYS][DH] fp32, 16 bytes per lane
    const long idx = PACKED ? ((long)hk * packed_blocks(p.packed, KEYS) + number) * np + part : (long)blockIdx.x * p.parts.partials() + p.parts.partial_of(kb, part);
    float* const base = p.partial + idx * 2 * KEYS * DH;
    if (has_cols) {
#pragma unroll
      for (int kbk = 0; kbk < KB; kbk++)
#pragma unroll
        for (int e4 = 0; e4 < 4; e4++) {
          float* const o = base + (long)(32 * kbk + kl) * DH + 32 * wave + 8 * e4 + 4 * g;
          *reinterpret_cast<f32x4*>(o) = f32x4{dkt[kbk][4 * e4], dkt[kbk][4 * e4 + 1], dkt[kbk][4 * e4 + 2], dkt[kbk][4 * e4 + 3]};
          *reinterpret_cast<f32x4*>(o + KEYS * DH) = f32x4{dvt[kbk][4 * e4], dvt[kbk][4 * e4 + 1], dvt[kbk][4 * e4 + 2], dvt[kbk][4 * e4 + 3]};
        }
    }
    __syncthreads();                                          // (the left waves count two barriers behind the loop)
    return;
  }
  // ---- dk = scale * dK^T transposed, dv = dV^T transposed, put together in LDS (the ring is free) and written as whole rows
  constexpr int EROW = DH * 2 + 16;
  lds_u8* const edk = lds;
  lds_u8* const edv = lds + KEYS * EROW;
  static_assert(2 * KEYS * EROW <= 3 * SLOT, "dK and dV tiles must fit in the ring");
  if (has_cols) {
#pragma unroll
    for (int kbk = 0; kbk < KB; kbk++)
#pragma unroll
      for (int e4 = 0; e4 < 4; e4++) {
        bf16x4 vk, vv;
#pragma unroll
        for (int r = 0; r < 4; r++) { vk[r] = (bf16_t)(dkt[kbk][4 * e4 + r] * p.scale); vv[r] = (bf16_t)dvt[kbk][4 * e4 + r]; }
        const int off = (32 * kbk + kl) * EROW + (32 * wave + 8 * e4 + 4 * g) * 2;
        *reinterpret_cast<LDS_AS bf16x4*>(edk + off) = vk;
        *reinterpret_cast<LDS_AS bf16x4*>(edv + off) = vv;
      }
  }
  __syncthreads();
  {
    constexpr int LPR = DH / 8, RPI = 64 / LPR;               // lanes per row, rows per wave-wide store
    const int rl = lane / LPR, piece = lane % LPR;
#pragma unroll
    for (int r0 = 0; r0 < KEYS / 4; r0 += RPI) {
      const int row = KEYS / 4 * wave + r0 + rl;              // this wave's quarter of the key rows
      const int krow = kv0 + row;
      if (krow < S) {
        bf16_t* const out = p.dqkv + (tok0 + krow) * p.ld_dqkv + (long)(p.H + hk) * DH + 8 * piece;
        *reinterpret_cast<u32x4*>(out) = *reinterpret_cast<const LDS_AS u32x4*>(edk + row * EROW + 16 * piece);
        *reinterpret_cast<u32x4*>(out + (long)p.KV * DH) = *reinterpret_cast<const LDS_AS u32x4*>(edv + row * EROW + 16 * piece);
      }
    }
  }
}

// dk and dv of the key blocks that were cut: the parts added up in order.  One workgroup = 8 or 16 key rows of one of them; a thread has 8
// columns of one row of dK or dV.  Bound by the latency of the parts: 38 of them 13.4 us one at a time, 7.6 eight at a time.
template <int DH, int KEYS, int PACKED>
__global__ __launch_bounds__(256) void window_bwd_join_kernel(WinKvParams p) {
  constexpr int LPR = DH / 8, ROWS = 256 / (2 * LPR);
  const int per = KEYS / ROWS, cut = (PACKED ? (int)blockIdx.x / p.KV : (int)blockIdx.y) / per;
  const int number = !PACKED && p.parts.sink_parts == 1 ? cut + p.parts.sink_blocks : cut;       // (blocks that are cut: the sinks', the others', or all)
  const int b = PACKED ? 0 : (int)blockIdx.x / p.KV, hk = (int)blockIdx.x % p.KV;
  SeqOf seq{(long)b * p.S, 0, p.S, number};
  if constexpr (PACKED) seq = SeqOf::of<PACKED, KEYS, false>(p.packed, number);
  const int kb = seq.block;
  const int which = (int)threadIdx.x / (ROWS * LPR), t = (int)threadIdx.x % (ROWS * LPR);
  const int row = ((PACKED ? (int)blockIdx.x / p.KV : (int)blockIdx.y) % per) * ROWS + t / LPR, col = 8 * (t % LPR);
  const int np = !PACKED && kb < p.parts.sink_blocks ? p.parts.sink_parts : p.parts.other_parts;
  const long first = PACKED ? ((long)hk * packed_blocks(p.packed, KEYS) + number) * np : (long)blockIdx.x * p.parts.partials() + p.parts.partial_of(kb, 0);
  const int krow = kb * KEYS + row;
  if (krow >= seq.S) return;
  const float* src = p.partial + first * 2 * KEYS * DH + (long)which * KEYS * DH + (long)row * DH + col;
  constexpr long PART = 2L * KEYS * DH;
  constexpr int AT_ONCE = 8;                         // parts on their way together
  float v[8] = {};
  int i = 0;
  for (; i + AT_ONCE <= np; i += AT_ONCE) {
    f32x4 a[AT_ONCE][2];
#pragma unroll
    for (int j = 0; j < AT_ONCE; j++)
#pragma unroll
      for (int h = 0; h < 2; h++) a[j][h] = *reinterpret_cast<const f32x4*>(src + (i + j) * PART + 4 * h);
#pragma unroll
    for (int j = 0; j < AT_ONCE; j++)
#pragma unroll
      for (int k = 0; k < 8; k++) v[k] += a[j][k >> 2][k & 3];
  }
  for (; i < np; i++)
#pragma unroll
    for (int k = 0; k < 8; k++) v[k] += src[i * PART + k];
#pragma unroll
  for (int k = 0; k < 8; k++) v[k] *= which ? 1.f : p.scale;
  Vec<bf16_t>::store(p.dqkv + (seq.tok0 + krow) * p.ld_dqkv + (long)(p.H + which * p.KV + hk) * DH + col, v);
}

// ------------------------------------------------------------------------------------------ one new token per sequence
// Workgroup = one (sequence, key head, 32 query heads of its group) and a share of the keys that the new token sees, 4 waves that take
// tiles of 32 keys in turn, each through a ring of its own in LDS: no barrier before the waves join.  S^T = K Q^T with the query heads
// as columns (unused ones: zeros), then O^T += V^T P^T, as in the forward.  The share that is done last joins them all (a launch for it took
// 3.8 us, and its host side as much again).  Bound by the reading of K and V: a tile is 16 KiB at
// head_dim 128 and 16 MFMAs, a fifteenth of the time that it takes to arrive.  64 ragged sequences of up to 4100 seen keys, 8 heads of 128,
// 974 MB: 170 us, 5.7 TB/s; one sequence of 700 keys (2.9 MB) 8.9 us, of which a launch that reads nothing is 3.
// Seen keys are numbered v = 0 .. seen - 1: the sinks, then the window in order; number v lies in slot v (sinks) or
// sinks + (first + v - n_sink) mod ring.
struct WinDecodeParams {
  const bf16_t* q; long ld_q;          // [B, >= H*DH]
  const bf16_t* ck; const bf16_t* cv; long ld_c; long seq_stride;   // [B][capacity][>= KV*DH]
  const int* lengths;
  bf16_t* out; long ld_out;
  float* lse;                          // [B, H]
  float* part_o; float2* part_ml;      // [B, H, splits][DH], [B, H, splits] (splits > 1)
  unsigned* arrived;                   // [B, KV, 32-head groups]: shares that are done; zero before and after every call
  int B, H, KV, G, capacity, window, sinks, splits;
  float scale_log2e;
};

// Tiles of a share, at least: two per wave, at head_dim 64 four (us, 8 / 16 tiles: 300 keys at 64 8.3 / 7.0, 500 12.1 / 10.7; 700 at 128 9.0 / 11.5).
constexpr int share_tiles(int head_dim) { return 1024 / head_dim; }

// Numbers that another workgroup, perhaps on another XCD, reads behind a counter: written through to memory that all of them see, and read from
// there.  (A fence that writes the whole L2 back instead cost 40 to 80 us a call where many workgroups have one.)
__device__ __forceinline__ void store_shared(float* p, float a, float b) {
  const uint64_t v = (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a);
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_shared(const float* p) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Asynchronous global -> LDS copy of 16 bytes per lane from a 64-bit address (a cache may be longer than a buffer descriptor's range).
// PAST: not kept in the caches, for more keys than they hold (64 sequences of 4096 keys of 8 heads of 128 201 -> 183 us; 16.4 MB 11.5 -> 12.0).
template <bool PAST>
__device__ __forceinline__ void dma16_far(uint32_t lds_base, const void* src) {
  if constexpr (PAST) asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off nt" :: "s"(lds_base), "v"(src) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds_base), "v"(src) : "memory");
}

template <int DH, bool PAST>
__global__ __launch_bounds__(256) void window_decode_kernel(WinDecodeParams p) {
  using HT = HeadTile<DH>;
  constexpr int KS = DH / 16, DT = DH / 32, IMG = 32 * HT::RB, SLOT = 2 * IMG, NCH = IMG / 1024, RING = 2;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  const int lane = threadIdx.x & 63, ql = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  lds_u8* const lds = LDS_PTR(unsigned char, smem_raw) + wave * (RING * SLOT);
  const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)lds);
  const int b = (int)blockIdx.x / p.KV, hk = (int)blockIdx.x % p.KV, sp = (int)blockIdx.y, gq0 = (int)blockIdx.z * 32;
  const int nh = p.G - gq0 < 32 ? p.G - gq0 : 32;              // query heads of this workgroup
  const int h = hk * p.G + gq0 + ql;                           // this lane's (if ql < nh)
  const int len = __builtin_amdgcn_readfirstlane(p.lengths[b]);
  const int ring = p.capacity - p.sinks, reach = p.window < ring ? p.window : ring;
  const int n_sink = len < p.sinks ? (len > 0 ? len : 0) : p.sinks;
  const int first = len - reach > p.sinks ? len - reach : p.sinks;
  const int seen = n_sink + (len > first ? len - first : 0);
  const int r0 = (first - p.sinks) % ring;                     // ring place of the window's first key
  // shares of the tiles that there are: at most `splits`, none below share_tiles; the workgroups behind them have nothing to do
  const int tiles = (seen + 31) / 32, even = (tiles + p.splits - 1) / p.splits, per = even > share_tiles(DH) ? even : share_tiles(DH);
  const int shares = tiles > per ? (tiles + per - 1) / per : 1;
  if (sp >= shares) return;
  const int t0 = sp * per, t1 = t0 + per < tiles ? t0 + per : tiles;

  const typename HT::Offsets fo = HT::offsets(lane);
  bf16x8 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; s++) {
    qf[s] = bf16x8{};
    if (ql < nh) qf[s] = *reinterpret_cast<const bf16x8*>(p.q + (long)b * p.ld_q + (long)h * DH + 16 * s + 8 * g);
  }
  const bf16_t* const kbase = p.ck + (long)b * p.seq_stride + (long)hk * DH;
  const bf16_t* const vbase = p.cv + (long)b * p.seq_stride + (long)hk * DH;
  // (numbers past the last read the last key's row: finite, and their probability is zero)
  auto issue = [&](int t) {
    const uint32_t base = lds0 + (((t - t0) >> 2) & (RING - 1)) * SLOT;
#pragma unroll
    for (int c = 0; c < NCH; c++) {
      const int row = HT::RPC * c + lane / HT::GPRW, G16 = (lane % HT::GPRW) ^ HT::swz(row);
      int v = 32 * t + row;
      v = v < seen ? v : seen - 1;
      int x = r0 + v - n_sink;
      x = x >= ring ? x - ring : x;
      const long off = (long)(v < n_sink ? v : p.sinks + x) * p.ld_c + 8 * G16;
      dma16_far<PAST>(base + c * 1024, kbase + off);
      dma16_far<PAST>(base + IMG + c * 1024, vbase + off);
    }
  };
  f32x16 ot[DT];
#pragma unroll
  for (int t = 0; t < DT; t++)
#pragma unroll
    for (int e = 0; e < 16; e++) ot[t][e] = 0.f;
  float m = -INFINITY, l = 0.f;
  if (t0 + wave < t1) issue(t0 + wave);
  for (int t = t0 + wave; t < t1; t += 4) {
    if (t + 4 < t1) {
      issue(t + 4);
      wait_vmem<2 * NCH>();
    } else {
      wait_vmem<0>();
    }
    asm volatile("" ::: "memory");
    lds_u8* const kimg = lds + (((t - t0) >> 2) & (RING - 1)) * SLOT;
    lds_u8* const vimg = kimg + IMG;
    f32x16 st;
#pragma unroll
    for (int e = 0; e < 16; e++) st[e] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; s++) st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(HT::rows_frag(kimg, fo, 0, s), qf[s], st, 0, 0, 0);
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; e++) {
      if (32 * t + 32 > seen && 32 * t + 8 * (e >> 2) + (e & 3) + 4 * g >= seen) st[e] = -INFINITY;
      mx = fmaxf(mx, st[e]);
    }
    mx *= p.scale_log2e;
    const float mnew = fmaxf(m, fmaxf(mx, xor32(mx)));
    const float ref = mnew == -INFINITY ? 0.f : mnew, alpha = __builtin_amdgcn_exp2f(m - ref);
    m = mnew;
    l *= alpha;
#pragma unroll
    for (int e = 0; e < 16; e++) {
      st[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[e], p.scale_log2e, -ref));
      l += st[e];
    }
#pragma unroll
    for (int tt = 0; tt < DT; tt++)
#pragma unroll
      for (int e = 0; e < 16; e++) ot[tt][e] *= alpha;
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const bf16x8 pb = pack8(st, u);
#pragma unroll
      for (int tt = 0; tt < DT; tt++) ot[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(HT::cols_frag(vimg, fo, 0, u, tt), pb, ot[tt], 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // every fragment of the slot has been read before copies into it start
  }
  l += xor32(l);
  // ---- the four waves join (each leaves sums and statistics in its own part of the LDS, head by head)
  constexpr int OROW = DH + 4;                                 // floats of a head's row
  LDS_AS float* const mine = reinterpret_cast<LDS_AS float*>(lds);
  static_assert(32 * OROW * 4 + 256 <= RING * SLOT, "a wave's sums must fit in its ring");
#pragma unroll
  for (int t = 0; t < DT; t++)
#pragma unroll
    for (int e4 = 0; e4 < 4; e4++)
      *reinterpret_cast<LDS_AS f32x4*>(mine + ql * OROW + 32 * t + 8 * e4 + 4 * g) = f32x4{ot[t][4 * e4], ot[t][4 * e4 + 1], ot[t][4 * e4 + 2], ot[t][4 * e4 + 3]};
  if (g == 0) {
    mine[32 * OROW + ql] = m;
    mine[32 * OROW + 32 + ql] = l;
  }
  __syncthreads();
  LDS_AS float* const all = reinterpret_cast<LDS_AS float*>(LDS_PTR(unsigned char, smem_raw));
  auto finish = [&](int r, int c, f32x4 o, float M, float L) {  // columns c .. c + 3 of this workgroup's head r
    const long head = (long)b * p.H + hk * p.G + gq0 + r;
    const float inv = L > 0.f ? 1.f / L : 0.f;                 // (no key seen: zeros)
    bf16x4 v;
#pragma unroll
    for (int k = 0; k < 4; k++) v[k] = (bf16_t)(o[k] * inv);
    *reinterpret_cast<bf16x4*>(p.out + (long)b * p.ld_out + (long)(hk * p.G + gq0 + r) * DH + c) = v;
    if (c == 0) p.lse[head] = M + __builtin_amdgcn_logf(L);
  };
  constexpr int WSTRIDE = RING * SLOT / 4;
  for (int i = (int)threadIdx.x; i < nh * (DH / 4); i += 256) {
    const int r = i / (DH / 4), c = 4 * (i % (DH / 4));
    float mw[4], M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < 4; w++) {
      mw[w] = all[w * WSTRIDE + 32 * OROW + r];
      M = fmaxf(M, mw[w]);
    }
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; w++) {
      const float f = __builtin_amdgcn_exp2f(mw[w] - (M == -INFINITY ? 0.f : M));
      L += f * all[w * WSTRIDE + 32 * OROW + 32 + r];
      const f32x4 x = *reinterpret_cast<LDS_AS f32x4*>(all + w * WSTRIDE + r * OROW + c);
#pragma unroll
      for (int k = 0; k < 4; k++) o[k] += f * x[k];
    }
    const long head = (long)b * p.H + hk * p.G + gq0 + r;
    if (shares > 1) {
      float* const at = p.part_o + (head * p.splits + sp) * DH + c;
      store_shared(at, o[0], o[1]);
      store_shared(at + 2, o[2], o[3]);
      if (c == 0) store_shared(reinterpret_cast<float*>(p.part_ml + head * p.splits + sp), M, L);
    } else {
      finish(r, c, o, M, L);
    }
  }
  if (shares == 1) return;
  // ---- the share that is done last joins all of them, in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // this wave's sums are where everyone sees them ...
  __syncthreads();                                            // ... and every wave's, before the share is counted
  LDS_AS unsigned* const flag = reinterpret_cast<LDS_AS unsigned*>(all);
  if (threadIdx.x == 0) {
    unsigned* const count = p.arrived + ((long)blockIdx.z * gridDim.x + blockIdx.x);
    const bool last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == (unsigned)shares;
    if (last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *flag = last ? 1u : 0u;
  }
  __syncthreads();
  if (!*flag) return;
  for (int i = (int)threadIdx.x; i < nh * (DH / 4); i += 256) {
    const int r = i / (DH / 4), c = 4 * (i % (DH / 4));
    const long at = ((long)b * p.H + hk * p.G + gq0 + r) * p.splits;
    float M = -INFINITY, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int k = 0; k < shares; k++) {                         // (one pass: the loads of eight shares wait for memory together)
      const float2 ml = load_shared(reinterpret_cast<const float*>(p.part_ml + at + k));
      const float2 x = load_shared(p.part_o + (at + k) * DH + c), z = load_shared(p.part_o + (at + k) * DH + c + 2);
      const float m2 = fmaxf(M, ml.x), ref2 = m2 == -INFINITY ? 0.f : m2;
      const float f = __builtin_amdgcn_exp2f(ml.x - ref2), keep = __builtin_amdgcn_exp2f(M - ref2);
      M = m2;
      L = L * keep + f * ml.y;
      o[0] = o[0] * keep + f * x.x;
      o[1] = o[1] * keep + f * x.y;
      o[2] = o[2] * keep + f * z.x;
      o[3] = o[3] * keep + f * z.y;
    }
    finish(r, c, o, M, L);
  }
}

// ------------------------------------------------------------------------------------------ launches
template <int DH, bool AHEAD, int SPLIT, int HW = 1, int PACKED = 0>
static hipError_t launch_fwd(const WinParams& p, hipStream_t s) {
  constexpr size_t smem = 2 * 2 * 64 * DH * 2;
  auto kern = window_fwd_kernel<DH, AHEAD, SPLIT, HW, PACKED>;
  static AttrOnce once;
  if (hipError_t e = once.set(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  const dim3 grid = PACKED != 0 ? dim3((unsigned)(p.H / HW * packed_blocks(p.packed, 128 / SPLIT / HW))) : dim3((unsigned)(p.H * p.B), (unsigned)((p.S * SPLIT + 127) / 128));
  hipLaunchKernelGGL(kern, grid, dim3(256), smem, s, p);
  return hipGetLastError();
}

hipError_t window_attention_fwd(const WindowShape& w, const int* lengths, const void* qkv, long ld_qkv, void* out, long ld_out,
                                float* lse, hipStream_t s) {
  WinParams p{};
  p.qkv = (const bf16_t*)qkv; p.ld_qkv = ld_qkv; p.out = (bf16_t*)out; p.ld_out = ld_out; p.lse = lse; p.lengths = lengths;
  p.B = w.batch; p.H = w.heads; p.KV = w.kv_heads; p.G = w.heads / w.kv_heads; p.S = w.seq; p.window = w.window; p.sinks = w.sinks;
  p.scale_log2e = 1.4426950408889634f / sqrtf((float)w.head_dim);
  const long groups = (long)w.batch * w.heads * ((w.seq + 127) / 128);
  // 64 queries per workgroup where those of 128 leave compute units short of work; a unit has room for 2 workgroups at head_dim 128, 4 at 64.  us, 128 / 64
  // queries: 8 heads of 128, 700 tokens, window 300 16.2 / 10.3; 32, 1024, 256 17.3 / 13.8; 40, 512, all 16.1 / 13.3, but 32, 2048, 512 28.5 / 31.0; of 64:
  // 12 heads, 4 ragged sequences of 1001, 300 15.7 / 11.8; 16, 4096, all 61.8 / 55.6, but 32, 4 of 2048, 256 38.4 / 39.9
  if (w.seq > 64 && groups <= (w.head_dim == 64 ? 512 : 256)) return w.head_dim == 128 ? launch_fwd<128, false, 2>(p, s) : launch_fwd<64, false, 2>(p, s);
  // the scores of the next block ahead of its turn (AHEAD) / not: 32 heads of 128, 2 sequences of 4096, window 64 54.6 / 52.5, 128 68.5 / 65.3, 256 71.8 /
  // 71.3, one of 8192, 512 107.7 / 104.4, 2048 247.9 / 250.4, 2 of 8192, all 963 / 970.  At head_dim 64 its registers leave a unit 3 workgroups of 4: 16 heads, 2
  // of 4096, 1024 53.2 / 47.2, 32 heads, 4 of 4096, all 302 / 293, but 16 heads, 2 of 4096, all 82.6 / 87.9
  if (w.head_dim == 64) return launch_fwd<64, false, 1>(p, s);
  return w.seq <= 256 || w.window <= 512 ? launch_fwd<128, false, 1>(p, s) : launch_fwd<128, true, 1>(p, s);
}

template <int DH, int SPLIT, int HW = 1, int PACKED = 0>
static hipError_t launch_dq(const WinDqParams& p, hipStream_t s) {
  constexpr size_t smem = 2 * 2 * 64 * DH * 2;
  auto kern = window_bwd_dq_kernel<DH, SPLIT, HW, PACKED>;
  static AttrOnce once;
  if (hipError_t e = once.set(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  const dim3 grid = PACKED != 0 ? dim3((unsigned)(p.H / HW * packed_blocks(p.packed, 128 / SPLIT / HW))) : dim3((unsigned)(p.H * p.B), (unsigned)((p.S * SPLIT + 127) / 128));
  hipLaunchKernelGGL(kern, grid, dim3(256), smem, s, p);
  return hipGetLastError();
}

template <int DH, int KEYS, int PACKED = 0>
static hipError_t launch_kv(const WinKvParams& p, hipStream_t s) {
  constexpr size_t smem = 3 * (2 * 64 * DH * 2 + (DH == 64 ? 0 : 1024)) + 2 * 4 * 4096;       // three slots, two hand-over buffers
  auto kern = window_bwd_kv_kernel<DH, KEYS, PACKED>;
  static AttrOnce once;
  if (hipError_t e = once.set(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  constexpr int per = KEYS / (256 / (2 * (DH / 8)));
  if constexpr (PACKED != 0) {
    const long blocks = p.KV * packed_blocks(p.packed, KEYS);
    hipLaunchKernelGGL(kern, dim3((unsigned)(blocks * p.parts.other_parts)), dim3(512), smem, s, p);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || p.parts.other_parts == 1) return e;
    hipLaunchKernelGGL((window_bwd_join_kernel<DH, KEYS, PACKED>), dim3((unsigned)(blocks * per)), dim3(256), 0, s, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(kern, dim3((unsigned)(p.KV * p.B), (unsigned)p.parts.workgroups()), dim3(512), smem, s, p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || !p.parts.cut_blocks()) return e;
  hipLaunchKernelGGL((window_bwd_join_kernel<DH, KEYS, 0>), dim3((unsigned)(p.KV * p.B), (unsigned)(p.parts.cut_blocks() * per)), dim3(256), 0, s, p);
  return hipGetLastError();
}

WindowParts window_parts(const WindowShape& w) {
  WindowParts r{};
  const long heads = (long)w.batch * w.kv_heads;
  // 64 keys to a block at head_dim 64, where two such workgroups fit a compute unit; at 128 on few blocks, which are cut into parts of half the partial
  // sums then or into none, and for short windows, of which a block of 128 sees more than it is seen by.  us of the backward, 128 / 64: 8 key heads of 128,
  // 1024 tokens, window 256 61.3 / 48.0, 2048, 512 105.9 / 88.3, 8192, 512 369 / 334, 2 sequences of 4096, 128 207 / 182, but 1024 472 / 477, and 8192,
  // 2048 846 / 871; 16 heads of 64, 2 sequences of 4096, all 315 / 288, window 1024 171 / 156; 4 ragged ones of 1001, 4 heads, 300 42.4 / 35.3.
  r.keys = w.head_dim == 64 || heads * ((w.seq + 127) / 128) <= 256 || w.window <= 768 ? 64 : 128;
  r.blocks = (w.seq + r.keys - 1) / r.keys;
  const int sinks = w.sinks < w.seq ? w.sinks : w.seq, G = w.heads / w.kv_heads;
  r.sink_blocks = (sinks + r.keys - 1) / r.keys;
  const long all = (w.seq + 63) / 64, seen = ((long)w.window + r.keys - 2 + 64) / 64 + 1;
  const long sink_pairs = G * all, other_pairs = G * (seen < all ? seen : all);      // pairs of the longest lists, of each kind
  // a part: enough of them for 256 workgroups (for 512, 4 ragged sequences of 1001, 4 key heads of 64 42 us for 35), where the lists are long enough for that (4 pairs
  // each; 6, 8 and 12 took the same time), at most a whole list of the other blocks;
  // of the sinks' lists, so that they make no more than 1024 parts in all (sinks may be as many as tokens, and the window short)
  const long others = r.blocks - r.sink_blocks;
  const long pairs = heads * (r.sink_blocks * sink_pairs + others * other_pairs);
  long share = other_pairs * (heads * r.blocks < 256 ? heads * r.blocks : 256) / 256;
  share = share < 4 ? 4 : share;
  share = share > other_pairs ? other_pairs : share;
  r.other_parts = (int)((other_pairs + share - 1) / share);
  const long sink_share = share > (pairs + 1023) / 1024 ? share : (pairs + 1023) / 1024;
  r.sink_parts = (int)((sink_pairs + sink_share - 1) / sink_share);
  return r;
}

size_t window_attention_p1_partial_bytes(const WindowShape& w) {
  const WindowParts r = window_parts(w);
  return (size_t)w.batch * w.kv_heads * r.partials() * 2 * r.keys * w.head_dim * sizeof(float);
}

hipError_t window_attention_p1(const WindowShape& w, const int* lengths, const void* qkv, long ld_qkv, const void* out,
                               const void* d_out, long ld_out, const float* lse, void* dqkv, long ld_dqkv, float* delta,
                               float* partial, hipStream_t s) {
  WinDqParams q{};
  q.qkv = (const bf16_t*)qkv; q.ld_qkv = ld_qkv; q.dout = (const bf16_t*)d_out; q.out = (const bf16_t*)out; q.ld_do = ld_out;
  q.lse = lse; q.delta = delta; q.lengths = lengths; q.dqkv = (bf16_t*)dqkv; q.ld_dqkv = ld_dqkv;
  q.B = w.batch; q.H = w.heads; q.KV = w.kv_heads; q.G = w.heads / w.kv_heads; q.S = w.seq; q.window = w.window; q.sinks = w.sinks;
  q.scale = 1.f / sqrtf((float)w.head_dim);
  q.scale_log2e = 1.4426950408889634f * q.scale;
  // 64 queries per workgroup as in the forward.  us of the whole backward, 128 / 64 queries of dq: 8 heads of 128, 700 tokens, window 300 33.4 / 26.9; 32, 1024, 256
  // 49.6 / 47.2; 40, 1024, 256 54.6 / 56.9; 32, 2 of 2048, 256 125.7 / 127.9; of 64: 12 heads, 4 ragged sequences of 1001, 300 39.0 / 36.7; 16, 4096, all 188 / 176; 32, 2
  // of 1024, all 78.2 / 76.3; 2048, 256 52.2 / 53.1; 4 of 2048, 256 120.8 / 126.5
  const long groups = (long)w.batch * w.heads * ((w.seq + 127) / 128);
  hipError_t e;
  if (groups <= (w.head_dim == 64 ? 512 : 256)) e = w.head_dim == 128 ? launch_dq<128, 2>(q, s) : launch_dq<64, 2>(q, s);
  else e = w.head_dim == 128 ? launch_dq<128, 1>(q, s) : launch_dq<64, 1>(q, s);
  if (e != hipSuccess) return e;
  WinKvParams p{};
  p.qkv = q.qkv; p.ld_qkv = ld_qkv; p.dout = q.dout; p.ld_do = ld_out; p.lse = lse; p.delta = delta; p.lengths = lengths;
  p.dqkv = q.dqkv; p.ld_dqkv = ld_dqkv; p.partial = partial;
  p.B = q.B; p.H = q.H; p.KV = q.KV; p.G = q.G; p.S = q.S; p.window = q.window; p.sinks = q.sinks;
  p.parts = window_parts(w);
  p.scale = q.scale; p.scale_log2e = q.scale_log2e;
  if (w.head_dim == 64) return launch_kv<64, 64>(p, s);
  return p.parts.keys == 64 ? launch_kv<128, 64>(p, s) : launch_kv<128, 128>(p, s);
}

// ---- packed sequences: the same kernels, by rules on the mean length, since the lengths are on the device
static Packed packed_of(const PackedShape& w) { return Packed{w.starts, w.seqs, w.rows}; }

// Whether blocks come the most work first whatever their sequence, or by their rows.  The last workgroups then are short ones; but a block has to be found among its
// sequences (0.95 us of each, of 5 sequences, by rows 0.5), and keys and values are met again later.  A rule of the launch, which does not know the lengths: with both orders in one kernel
// it was 4 % slower.
// Blocks of queries, `hw` heads to a workgroup: where an XCD has one group of heads (ids go round the 8 of them), keys and values are 32 MiB at most, and sequences few: up to 24 where
// two XCDs share a group or the workgroups are two and a half rounds of the card's places, else up to 8.  us of the forward, in order / the most first, lengths all alike and up to 30 times apart.
// Of 128, 16 heads on 8, 8192 rows: 8 sequences 55 / 48 and 77 / 67, 24 34 / 36 and 43 / 39; 16 on 4: 12 42 / 38 and 63 / 55; 32 on 8, 4096 rows: 5 45 / 41 and
// 75 / 73, 12 29 / 30 and 40 / 39; more rounds: 32 on 8, 8192 rows: 5 131 / 129 and 260 / 257, 8 94 / 93 and 134 / 132, but 12 75 / 79 and 84 / 89, 24 54 / 62 and 71 / 74; 32 on 4: 24 56 / 64 and 71 / 74; two XCDs to a group: 16 on 2,
// 16384 rows, 24 77 / 80 and 126 / 119; 8 on 1, 32768 rows: 12 209 / 193 and 317 / 295, 24 119 / 117 and 184 / 175.
// More groups: 64 on 8, 4096 rows: 5 80 / 85 and 91 / 96; 64 on 16: 8 63 / 73 and 84 / 86.  At 32 MiB, lengths apart: 8 on 1, 65536 rows, 5 and 20 1947 / 1948 and
// 972 / 987; 32 on 4, 16384 651 / 656 and 221 / 227.  Of 64, 32 on 8, 8192 rows: 8 52 / 47 and 91 / 82, 24 27 / 29 and 43 / 39; 16384 rows: 8 173 / 161 and 215 / 200, 32 63 / 66 and 84 / 88.
static bool queries_by_work(const PackedShape& w, int hw) {
  const long groups = w.heads / hw, workgroups = groups * ((long)w.rows * hw / 128 + w.seqs), places = w.head_dim == 64 ? 1024 : 512;
  return hw > 1 && w.seqs > 1 && groups <= 8 && (long)w.kv_heads * w.rows * w.head_dim <= 1 << 23 && w.seqs <= (groups <= 4 || 2 * workgroups <= 5 * places ? 24 : 8);
}
// Blocks of keys.  us of the backward, in order / the most first, lengths as above.  Of 128, 32 heads on 8: 8 sequences of 4096 rows in all 111 / 97 alike, 16 of 4000 80 / 75 and 107 / 98, 64 of
// 12800 262 / 247 and 288 / 277, but 64 of 8192 120 / 130 and 165 / 159 (alike and of 128 tokens the slower side, accepted for the others); 24 on 8: 48 of 8192
// 135 / 130 and 158 / 149, but 64 110 / 118 and 150 / 151; 8 on 8: 6 of 8192 136 / 123 and 189 / 177, but 16 75 / 78 and 101 / 104, 64 66 / 77 and 85 / 87; 16 on 16:
// 4 of 4096 103 / 96 and 136 / 133, but 16 of 8192 136 / 152 and 188 / 199; 32 on 16: 48 of 8192 159 / 183 and 192 / 206.  Of 64, 32 on 8: 32 of 8192 84 / 81 and 141 / 114, 64 of 16384
// 151 / 152 and 245 / 224; 16 on 8: 48 113 / 115 and 144 / 141, but 64 96 / 104 and 142 / 137; below 192 tokens on average 32 on 8, 64 of 8192 68 / 71 alike; 12 on 4, 30 of 67 24.4 / 26.2.
static bool keys_by_work(const PackedShape& w) {
  const int G = w.heads / w.kv_heads, most = G == 1 || w.kv_heads > 8 ? 8 : G < 4 ? 48 : 64;
  return w.seqs <= most && (w.head_dim == 128 || w.rows >= 192 * w.seqs);
}

template <int N> using Int = std::integral_constant<int, N>;

// Keys to a block and parts of a block's list of (query head, query step) pairs.
static WindowParts packed_parts(const PackedShape& w) {
  WindowParts r{};
  const int seqs = w.seqs > 0 ? w.seqs : 1, G = w.heads / w.kv_heads, mean = (w.rows + seqs - 1) / seqs;
  r.keys = w.head_dim == 64 || (long)w.kv_heads * (w.rows / 128 + seqs) <= 256 || mean <= 768 ? 64 : 128;
  const long blocks = (long)w.kv_heads * (w.rows / r.keys + seqs), pairs = (long)G * ((mean + 63) / 64), slots = w.head_dim == 64 ? 512 : 256;
  // a workgroup for every compute unit, with 4 pairs at least; two for every place, since the lists of a sequence are of all lengths from the longest down, where that
  // leaves 16 pairs.  us of the backward, one / two: 32 heads on 8 of 128, 2048 tokens 184 / 158, but 700 43.0 / 52.7; of 64: 16 on 4, 16 sequences of 8192 in all
  // 230 / 174, 32 on 8, 4096 336 / 305, but 12 on 4, 61 sequences of 67 on average 37.0 / 64.5
  long parts = (256 + blocks - 1) / blocks, more = (2 * slots + blocks - 1) / blocks;
  parts = parts < (pairs + 3) / 4 ? parts : (pairs + 3) / 4;
  more = more < pairs / 16 ? more : pairs / 16;
  parts = parts > more ? parts : more;
  r.other_parts = (int)parts;
  return r;
}

PackedPlan packed_plan(const PackedShape& w) {
  const int G = w.heads / w.kv_heads, heads = G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1, mean = w.rows / (w.seqs > 0 ? w.seqs : 1);
  const WindowParts keys = packed_parts(w);
  PackedPlan p{heads, 1, 0, 0, keys.keys, keys.other_parts, keys_by_work(w)};
  // 64 (query, head) rows to a workgroup where those of 128 leave compute units short of work, as for windows
  if (w.heads * ((long)w.rows / 128 + w.seqs) <= (w.head_dim == 64 ? 512 : 256)) {
    p.query_heads = heads < 2 ? 1 : 2;
    p.key_shares = 2;
    return p;
  }
  // scores ahead where sequences have several blocks of keys: us, ahead / not, 32 heads on 8 of 128: 5 sequences of 1639 141 / 149, 16 on 16, 6 of 683 on average 48 / 53,
  // 60 of 130 67 / 67
  p.scores_ahead = w.head_dim == 128 && mean > 256;
  p.queries_most_first = queries_by_work(w, heads);
  return p;
}

size_t packed_attention_p1_partial_bytes(const PackedShape& w) {
  const WindowParts r = packed_parts(w);
  return r.other_parts == 1 ? 0 : (size_t)w.kv_heads * packed_blocks(packed_of(w), r.keys) * r.other_parts * 2 * r.keys * w.head_dim * sizeof(float);
}

// run(head_dim, query heads of a workgroup)
template <typename F> static hipError_t by_heads(const PackedShape& w, const PackedPlan& plan, F run) {
  if (w.head_dim == 64) return plan.query_heads == 4 ? run(Int<64>(), Int<4>()) : plan.query_heads == 2 ? run(Int<64>(), Int<2>()) : run(Int<64>(), Int<1>());
  return plan.query_heads == 4 ? run(Int<128>(), Int<4>()) : plan.query_heads == 2 ? run(Int<128>(), Int<2>()) : run(Int<128>(), Int<1>());
}

hipError_t packed_attention_fwd(const PackedShape& w, const void* qkv, long ld_qkv, void* out, long ld_out, float* lse, hipStream_t s) {
  WinParams p{};
  p.qkv = (const bf16_t*)qkv; p.ld_qkv = ld_qkv; p.out = (bf16_t*)out; p.ld_out = ld_out; p.lse = lse; p.packed = packed_of(w);
  p.B = 1; p.H = w.heads; p.KV = w.kv_heads; p.G = w.heads / w.kv_heads; p.S = w.rows;
  p.scale_log2e = 1.4426950408889634f / sqrtf((float)w.head_dim);
  const PackedPlan plan = packed_plan(w);
  return by_heads(w, plan, [&](auto dh, auto hw) {
    constexpr int DH = decltype(dh)::value, HW = decltype(hw)::value;
    if constexpr (HW < 4) if (plan.key_shares == 2) return launch_fwd<DH, false, 2, HW, kInOrder>(p, s);
    if constexpr (DH == 128 && HW > 1) if (plan.scores_ahead && plan.queries_most_first) return launch_fwd<DH, true, 1, HW, kMostFirst>(p, s);
    if constexpr (DH == 128) if (plan.scores_ahead) return launch_fwd<DH, true, 1, HW, kInOrder>(p, s);
    if constexpr (HW > 1) if (plan.queries_most_first) return launch_fwd<DH, false, 1, HW, kMostFirst>(p, s);
    return launch_fwd<DH, false, 1, HW, kInOrder>(p, s);
  });
}

hipError_t packed_attention_p1(const PackedShape& w, const void* qkv, long ld_qkv, const void* out, const void* d_out, long ld_out, const float* lse,
                               void* dqkv, long ld_dqkv, float* delta, float* partial, hipStream_t s) {
  WinDqParams q{};
  q.qkv = (const bf16_t*)qkv; q.ld_qkv = ld_qkv; q.dout = (const bf16_t*)d_out; q.out = (const bf16_t*)out; q.ld_do = ld_out;
  q.lse = lse; q.delta = delta; q.packed = packed_of(w); q.dqkv = (bf16_t*)dqkv; q.ld_dqkv = ld_dqkv;
  q.B = 1; q.H = w.heads; q.KV = w.kv_heads; q.G = w.heads / w.kv_heads; q.S = w.rows;
  q.scale = 1.f / sqrtf((float)w.head_dim);
  q.scale_log2e = 1.4426950408889634f * q.scale;
  const PackedPlan plan = packed_plan(w);
  hipError_t e = by_heads(w, plan, [&](auto dh, auto hw) {
    constexpr int DH = decltype(dh)::value, HW = decltype(hw)::value;
    if constexpr (HW < 4) if (plan.key_shares == 2) return launch_dq<DH, 2, HW, kInOrder>(q, s);
    if constexpr (HW > 1) if (plan.queries_most_first) return launch_dq<DH, 1, HW, kMostFirst>(q, s);
    return launch_dq<DH, 1, HW, kInOrder>(q, s);
  });
  if (e != hipSuccess) return e;
  WinKvParams p{};
  p.qkv = q.qkv; p.ld_qkv = ld_qkv; p.dout = q.dout; p.ld_do = ld_out; p.lse = lse; p.delta = delta; p.packed = q.packed;
  p.dqkv = q.dqkv; p.ld_dqkv = ld_dqkv; p.partial = partial;
  p.B = 1; p.H = q.H; p.KV = q.KV; p.G = q.G; p.S = q.S;
  p.parts = packed_parts(w);
  p.scale = q.scale; p.scale_log2e = q.scale_log2e;
  auto run = [&](auto order) {
    constexpr int PACKED = decltype(order)::value;
    if (w.head_dim == 64) return launch_kv<64, 64, PACKED>(p, s);
    return p.parts.keys == 64 ? launch_kv<128, 64, PACKED>(p, s) : launch_kv<128, 128, PACKED>(p, s);
  };
  return plan.keys_most_first ? run(Int<kMostFirst>()) : run(Int<kInOrder>());
}

// Shares of a head's keys, at most: as many as make the rounds of workgroups (one per compute unit at head_dim 128, two at 64) short by this model, whose
// times, in us, are those of a tile in a workgroup when the chip is full, of one that has it to itself (the latency of its copies), and of a share's
// start and end.  They are those of head_dim 128; only their proportions matter, which half the bytes per tile and twice the workgroups per compute unit
// leave as they are: of 1, 2, 3, 4, 6, 8, 12, 16, 24 or 32 shares the model's are within 2 % of the fastest at both from 1000 keys on, us, one share / the model's / the fastest,
// 8 key heads of 128, 4 query heads each: 1 sequence of 4096 keys 56.3 / 10.7 / 10.6, 8 76.3 / 30.5 / 30.7, 12 78.2 / 47.7 / 47.5, 20 81.6 / 69.7 / 69.7, 33
// 147.6 / 122.0 / 121.6, 64 174.2 / 174.6 / 174.2, 5 of 16384 keys 96 / 68 (as many as leave no compute unit without one / the model's); of 64: 1 38.3 / 9.6 / 9.5,
// 8 47.3 / 16.9 / 16.8, 12 56.4 / 24.6 / 25.6, 20 59.3 / 34.8 / 34.7, 33 71.2 / 60.8 / 61.0, 64 89.6 / 89.6 / 89.6.  Lengths are not known here: all are taken for the
// longest (20 ragged ones 54.1, where as many as leave no compute unit without one take 48.2), and a cache that keeps less than the window for the window.
// A share costs the joining workgroup as much as most of a tile of keys (its sums of 32 heads, in proportion less of fewer), so no more than make the
// reading of a share and the joining of all of them about equal.  That is coarse where it binds: 32 query heads on one key head of 128, 300 keys in two shares 11.5, in
// one 8.7; 4096 in twelve 19.5, in sixteen 15.8 (whose tiles are two for every wave); 4 query heads, 300 keys 8.2, 7.7.  Nor more than eight rounds of workgroups (64
// sequences of 4096 keys in eight shares 235, in one 174) or 64 shares, which bounds the workspace.
int window_decode_splits(int batch, int heads, int kv_heads, int head_dim, long most_seen) {
  constexpr float kFull = 0.74f, kAlone = 0.44f, kStart = 4.f;
  const int group = heads / kv_heads, nh = group < 32 ? group : 32;
  const long groups = (long)batch * kv_heads * ((group + 31) / 32), tiles = (most_seen + 31) / 32, slots = head_dim == 64 ? 512 : 256;
  long most = (tiles + share_tiles(head_dim) - 1) / share_tiles(head_dim);
  const long level = (long)sqrt(40.0 * tiles / nh), some = 8 * slots / groups;
  most = most < level ? most : level;
  most = most < some ? most : some;
  most = most < 64 ? most : 64;
  int splits = 1;
  float best = 0.f;
  for (int n = 1; n == 1 || n <= most; n++) {
    const long rounds = groups * n / slots, rest = groups * n % slots, share = (tiles + n - 1) / n;
    const float last = kAlone + (kFull - kAlone) * (float)rest / (float)slots;
    const float us = rounds * (share * kFull + kStart) + (rest ? share * last + kStart : 0.f);
    if (n == 1 || us < 0.99f * best) { best = us; splits = n; }
  }
  return splits;
}

template <int DH, bool PAST>
static hipError_t launch_decode(const WinDecodeParams& p, hipStream_t s) {
  constexpr size_t smem = 4 * 2 * 2 * 32 * DH * 2;
  auto kern = window_decode_kernel<DH, PAST>;
  static AttrOnce once;
  if (hipError_t e = once.set(reinterpret_cast<const void*>(kern), smem); e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)(p.B * p.KV), (unsigned)p.splits, (unsigned)((p.G + 31) / 32)), dim3(256), smem, s, p);
  return hipGetLastError();
}

hipError_t window_decode(const WindowShape& w, int capacity, const int* lengths, const void* q, long ld_q, const void* cache_k,
                         const void* cache_v, long ld_cache, void* out, long ld_out, float* lse, int splits, unsigned* arrived,
                         float* part_o, float2* part_ml, hipStream_t s) {
  WinDecodeParams p{};
  p.q = (const bf16_t*)q; p.ld_q = ld_q; p.ck = (const bf16_t*)cache_k; p.cv = (const bf16_t*)cache_v; p.ld_c = ld_cache;
  p.seq_stride = (long)capacity * ld_cache;
  p.lengths = lengths; p.out = (bf16_t*)out; p.ld_out = ld_out; p.lse = lse; p.part_o = part_o; p.part_ml = part_ml; p.arrived = arrived;
  p.B = w.batch; p.H = w.heads; p.KV = w.kv_heads; p.G = w.heads / w.kv_heads; p.capacity = capacity; p.window = w.window;
  p.sinks = w.sinks; p.splits = splits;
  p.scale_log2e = 1.4426950408889634f / sqrtf((float)w.head_dim);
  // keys and values that the calls of these sizes may read, at most: more than the second-level caches hold?
  const long most = w.window + (long)w.sinks, rows = most < capacity ? most : capacity;
  if (4L * w.batch * w.kv_heads * rows * w.head_dim > (64L << 20)) return w.head_dim == 128 ? launch_decode<128, true>(p, s) : launch_decode<64, true>(p, s);
  return w.head_dim == 128 ? launch_decode<128, false>(p, s) : launch_decode<64, false>(p, s);
}

}  // namespace tbp
