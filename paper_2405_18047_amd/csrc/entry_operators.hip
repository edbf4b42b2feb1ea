// C entry points of the operators around a stage (long contexts, the last stage and serving; packed documents and a stash in 8 bits): argument
// checks, then the launches.
#include "entry.h"
#include "kernels.h"

using tbp::align_up;
using tbp::fail;

namespace {

hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }
bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

tbp_status check_storage(int dtype) {
  return dtype == TBP_F32 || dtype == TBP_BF16 ? TBP_OK : fail(TBP_EINVAL, "dtype must be TBP_F32 or TBP_BF16");
}

tbp_status check_heads(int n_heads, int n_kv_heads, int head_dim) {
  if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads) return fail(TBP_EINVAL, "n_kv_heads must divide n_heads");
  if (head_dim < 1 || (long)n_heads * head_dim >= (1L << 22)) return fail(TBP_EINVAL, "bad head_dim");
  return TBP_OK;
}

tbp_status check_window(int dtype, int batch, int n_heads, int n_kv_heads, int seq, int head_dim, int window, int sinks) {
  if (dtype != TBP_BF16) return fail(TBP_EINVAL, "window attention is built for bf16 storage only");
  if (head_dim != 64 && head_dim != 128) return fail(TBP_EINVAL, "window attention needs head_dim 64 or 128");
  if (check_heads(n_heads, n_kv_heads, head_dim) != TBP_OK) return TBP_EINVAL;
  if (batch < 0 || seq < 0) return fail(TBP_EINVAL, "negative size");
  if (seq > (1 << 20)) return fail(TBP_EINVAL, "seq %d above the limit %d", seq, 1 << 20);
  if (window < 1 || sinks < 0) return fail(TBP_EINVAL, "window must be at least 1 and sinks at least 0");
  if ((long)batch * n_heads >= (1L << 23)) return fail(TBP_EINVAL, "batch * n_heads must be below 2^23");
  return TBP_OK;
}

tbp_status check_ld(const char* what, long ld, long columns) {
  if (ld < columns || ld % 8 || ld >= (1L << 22))
    return fail(TBP_EINVAL, "%s must cover the %ld columns, be a multiple of 8 and below 2^22", what, columns);
  return TBP_OK;
}

tbp::WindowShape window_shape(int batch, int n_heads, int n_kv_heads, int seq, int head_dim, int window, int sinks) {
  return tbp::WindowShape{batch, n_heads, n_kv_heads, seq, head_dim, window < seq ? window : seq, sinks < seq ? sinks : seq};
}

size_t delta_bytes(int batch, int n_heads, int seq) { return align_up((size_t)batch * seq * n_heads * sizeof(float), 256); }

}  // namespace

extern "C" {

// ---- sliding-window attention ------------------------------------------------------------------------------------------
tbp_status tbp_window_attention_fwd(int dtype, int batch, int n_heads, int n_kv_heads, int seq, int head_dim, int window,
                                    int sinks, const int32_t* lengths, const void* qkv, int ld_qkv, void* out, int ld_out,
                                    float* lse, void* stream) {
  if (check_window(dtype, batch, n_heads, n_kv_heads, seq, head_dim, window, sinks) != TBP_OK) return TBP_EINVAL;
  if (batch == 0 || seq == 0) return TBP_OK;
  if (!qkv || !out || !lse) return fail(TBP_EINVAL, "qkv, out and lse must be non-null");
  if (check_ld("ld_qkv", ld_qkv, ((long)n_heads + 2L * n_kv_heads) * head_dim) != TBP_OK) return TBP_EINVAL;
  if (check_ld("ld_out", ld_out, (long)n_heads * head_dim) != TBP_OK) return TBP_EINVAL;
  if (misaligned(qkv, 16) || misaligned(out, 16)) return fail(TBP_EINVAL, "qkv and out must be 16-byte aligned");
  TBP_HIP(tbp::window_attention_fwd(window_shape(batch, n_heads, n_kv_heads, seq, head_dim, window, sinks), lengths, qkv, ld_qkv,
                                    out, ld_out, lse, stream_of(stream)));
  return TBP_OK;
}

size_t tbp_window_attention_p1_scratch_bytes(int batch, int n_heads, int n_kv_heads, int seq, int head_dim, int window, int sinks) {
  if (batch < 1 || seq < 1 || check_window(TBP_BF16, batch, n_heads, n_kv_heads, seq, head_dim, window, sinks) != TBP_OK) return 0;
  return delta_bytes(batch, n_heads, seq) +
         tbp::window_attention_p1_partial_bytes(window_shape(batch, n_heads, n_kv_heads, seq, head_dim, window, sinks));
}

tbp_status tbp_window_attention_p1(int dtype, int batch, int n_heads, int n_kv_heads, int seq, int head_dim, int window,
                                   int sinks, const int32_t* lengths, const void* qkv, int ld_qkv, const void* out,
                                   const void* d_out, int ld_out, const float* lse, void* dqkv, int ld_dqkv, void* scratch,
                                   void* stream) {
  if (check_window(dtype, batch, n_heads, n_kv_heads, seq, head_dim, window, sinks) != TBP_OK) return TBP_EINVAL;
  if (batch == 0 || seq == 0) return TBP_OK;
  if (!qkv || !out || !d_out || !lse || !dqkv || !scratch) return fail(TBP_EINVAL, "null pointer");
  const long columns = ((long)n_heads + 2L * n_kv_heads) * head_dim;
  if (check_ld("ld_qkv", ld_qkv, columns) != TBP_OK || check_ld("ld_dqkv", ld_dqkv, columns) != TBP_OK) return TBP_EINVAL;
  if (check_ld("ld_out", ld_out, (long)n_heads * head_dim) != TBP_OK) return TBP_EINVAL;
  if (misaligned(qkv, 16) || misaligned(out, 16) || misaligned(d_out, 16) || misaligned(dqkv, 16) || misaligned(scratch, 256))
    return fail(TBP_EINVAL, "tensors must be 16-byte aligned, scratch 256-byte aligned");
  TBP_HIP(tbp::window_attention_p1(window_shape(batch, n_heads, n_kv_heads, seq, head_dim, window, sinks), lengths, qkv, ld_qkv, out,
                                   d_out, ld_out, lse, dqkv, ld_dqkv, static_cast<float*>(scratch),
                                   reinterpret_cast<float*>(static_cast<char*>(scratch) + delta_bytes(batch, n_heads, seq)),
                                   stream_of(stream)));
  return TBP_OK;
}

// The decode workspace: counters of finished shares (zero between calls), then the shares' sums and statistics.
struct DecodeSpace { int splits; size_t part_o, part_ml, bytes; };
static DecodeSpace decode_space(int batch, int n_heads, int n_kv_heads, int head_dim, int window, int sinks) {
  DecodeSpace d{};
  d.splits = tbp::window_decode_splits(batch, n_heads, n_kv_heads, head_dim, (long)window + sinks);
  const size_t parts = (size_t)batch * n_heads * d.splits, groups = (n_heads / n_kv_heads + 31) / 32;
  d.part_o = align_up((size_t)batch * n_kv_heads * groups * sizeof(unsigned), 256);
  d.part_ml = d.part_o + align_up(parts * head_dim * sizeof(float), 256);
  d.bytes = d.part_ml + parts * sizeof(float2);
  return d;
}

size_t tbp_window_decode_workspace_bytes(int batch, int n_heads, int n_kv_heads, int head_dim, int window, int sinks) {
  if (batch < 1 || check_window(TBP_BF16, batch, n_heads, n_kv_heads, 0, head_dim, window, sinks) != TBP_OK) return 0;
  const DecodeSpace d = decode_space(batch, n_heads, n_kv_heads, head_dim, window, sinks);
  return d.splits == 1 ? 0 : d.bytes;
}

tbp_status tbp_window_decode(int dtype, int batch, int n_heads, int n_kv_heads, int head_dim, int window, int sinks,
                             int capacity, const int32_t* lengths, const void* q, int ld_q, const void* cache_k,
                             const void* cache_v, int ld_cache, void* out, int ld_out, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (check_window(dtype, batch, n_heads, n_kv_heads, 0, head_dim, window, sinks) != TBP_OK) return TBP_EINVAL;
  if (capacity <= sinks) return fail(TBP_EINVAL, "capacity must be above sinks");
  if (capacity > (1 << 30)) return fail(TBP_EINVAL, "capacity above the limit %d", 1 << 30);
  if (batch == 0) return TBP_OK;
  if (!lengths || !q || !cache_k || !cache_v || !out || !lse) return fail(TBP_EINVAL, "null pointer");
  const long wq = (long)n_heads * head_dim;
  if (check_ld("ld_q", ld_q, wq) != TBP_OK || check_ld("ld_out", ld_out, wq) != TBP_OK) return TBP_EINVAL;
  if (check_ld("ld_cache", ld_cache, (long)n_kv_heads * head_dim) != TBP_OK) return TBP_EINVAL;
  if (misaligned(q, 16) || misaligned(cache_k, 16) || misaligned(cache_v, 16) || misaligned(out, 16))
    return fail(TBP_EINVAL, "tensors must be 16-byte aligned");
  const DecodeSpace d = decode_space(batch, n_heads, n_kv_heads, head_dim, window, sinks);
  if (d.splits > 1 && (!workspace || misaligned(workspace, 256) || workspace_bytes < d.bytes))
    return fail(TBP_EINVAL, "workspace must be 256-byte aligned and have %zu bytes", d.bytes);
  char* const ws = static_cast<char*>(d.splits > 1 ? workspace : nullptr);
  TBP_HIP(tbp::window_decode(tbp::WindowShape{batch, n_heads, n_kv_heads, 0, head_dim, window, sinks}, capacity, lengths, q, ld_q,
                             cache_k, cache_v, ld_cache, out, ld_out, lse, d.splits, reinterpret_cast<unsigned*>(ws),
                             reinterpret_cast<float*>(ws + d.part_o), reinterpret_cast<float2*>(ws + d.part_ml), stream_of(stream)));
  return TBP_OK;
}

// ---- rotary positions ------------------------------------------------------------------------------------------------------
size_t tbp_rotary_table_bytes(int n_pos, int rot_dim) {
  return n_pos > 0 && rot_dim > 1 ? (size_t)n_pos * (rot_dim / 2) * sizeof(float2) : 0;
}

tbp_status tbp_rotary_table(int n_pos, int rot_dim, float base, const tbp_rotary_scale* scale, void* table, void* stream) {
  if (n_pos < 1 || rot_dim < 2 || rot_dim % 2 || !(base > 0.f) || !table) return fail(TBP_EINVAL, "bad rotary table arguments");
  if (rot_dim > 4096) return fail(TBP_EINVAL, "rot_dim above the limit 4096");
  if ((long)n_pos * (rot_dim / 2) >= (1L << 32) - 256) return fail(TBP_EINVAL, "a table of 2^32 - 256 entries or more");      // (a launch's threads)
  if (misaligned(table, 8)) return fail(TBP_EINVAL, "table must be 8-byte aligned");
  tbp::RotaryScale sc{tbp::ROTARY_PLAIN, 1.f, 0.f, 1.f, 1.f, 1.f};
  if (scale) {
    if (scale->scaling < TBP_ROTARY_PLAIN || scale->scaling > TBP_ROTARY_RAMP) return fail(TBP_EINVAL, "unknown rotary scaling %d", scale->scaling);
    if (scale->scaling != TBP_ROTARY_PLAIN && !(scale->factor > 0.f)) return fail(TBP_EINVAL, "the scaling factor must be above 0");
    if (scale->scaling == TBP_ROTARY_BASE && rot_dim == 2) return fail(TBP_EINVAL, "a scaled base needs rot_dim above 2");
    if (scale->scaling == TBP_ROTARY_RAMP && (!(scale->low < scale->high) || !(scale->original > 0.f)))
      return fail(TBP_EINVAL, "a ramp needs low < high and an original context above 0");
    if (!(scale->magnitude >= 0.f)) return fail(TBP_EINVAL, "the magnitude must be at least 0");
    sc = tbp::RotaryScale{scale->scaling, scale->factor, scale->low, scale->high, scale->original, scale->magnitude == 0.f ? 1.f : scale->magnitude};
  }
  TBP_HIP(tbp::rotary_table(n_pos, rot_dim, base, sc, static_cast<float2*>(table), stream_of(stream)));
  return TBP_OK;
}

static tbp_status check_rotary(int dtype, int head_dim, int rot_dim, int layout, const void* table, int n_pos) {
  if (check_storage(dtype) != TBP_OK) return TBP_EINVAL;
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim) return fail(TBP_EINVAL, "rot_dim must be even, at least 2 and at most head_dim");
  if (layout != TBP_ROTARY_HALF && layout != TBP_ROTARY_INTERLEAVED) return fail(TBP_EINVAL, "unknown rotary layout %d", layout);
  if (n_pos < 1) return fail(TBP_EINVAL, "n_pos must be at least 1");
  if (!table || misaligned(table, 8)) return fail(TBP_EINVAL, "table must be non-null and 8-byte aligned");
  return TBP_OK;
}

tbp_status tbp_rotary(int dtype, int rows, int n_heads, int head_dim, int rot_dim, int layout, const void* table, int n_pos,
                      const int32_t* positions, int seq, int backward, const void* x, int ld_x, void* y, int ld_y, void* stream) {
  if (rows < 0 || n_heads < 0 || head_dim < 1) return fail(TBP_EINVAL, "negative size");
  if (check_rotary(dtype, head_dim, rot_dim, layout, table, n_pos) != TBP_OK) return TBP_EINVAL;
  if (!positions && seq < 1) return fail(TBP_EINVAL, "without positions seq must be at least 1");
  const long columns = (long)n_heads * head_dim;
  if (ld_x < columns || ld_y < columns) return fail(TBP_EINVAL, "leading dimensions must cover the %ld head columns", columns);
  if (rows == 0 || n_heads == 0) return TBP_OK;
  if (!x || !y) return fail(TBP_EINVAL, "null pointer");
  const size_t e = dtype == TBP_BF16 ? 2 : 4;
  if (misaligned(x, e) || misaligned(y, e)) return fail(TBP_EINVAL, "tensors must be aligned to their elements");
  if (x == y && ld_x != ld_y) return fail(TBP_EINVAL, "in place both leading dimensions must be the same");
  tbp::RotaryParams p{};
  p.x = x; p.ld_x = ld_x; p.y = y; p.ld_y = ld_y; p.table = static_cast<const float2*>(table); p.n_pos = n_pos;
  p.positions = positions; p.seq = seq < 1 ? 1 : seq; p.rows = rows; p.heads = n_heads; p.dh = head_dim; p.half = rot_dim / 2;
  p.interleaved = layout; p.sgn = backward ? -1.f : 1.f;
  TBP_HIP(tbp::rotary(dtype, p, stream_of(stream)));
  return TBP_OK;
}

tbp_status tbp_rotary_append(int dtype, int batch, int n_new, int n_heads, int n_kv_heads, int head_dim, int rot_dim, int layout,
                             const void* table, int n_pos, const int32_t* lengths, const void* qkv, int ld_qkv, void* q_out,
                             int ld_q, void* cache_k, void* cache_v, int ld_cache, int capacity, int sinks, void* stream) {
  if (check_heads(n_heads, n_kv_heads, head_dim) != TBP_OK) return TBP_EINVAL;
  if (check_rotary(dtype, head_dim, rot_dim, layout, table, n_pos) != TBP_OK) return TBP_EINVAL;
  if (batch < 0 || n_new < 0) return fail(TBP_EINVAL, "negative size");
  if ((long)batch * n_new > 0x7fffffffL) return fail(TBP_EINVAL, "batch * n_new too large");
  if (sinks < 0 || capacity <= sinks) return fail(TBP_EINVAL, "capacity must be above sinks, sinks at least 0");
  const long wq = (long)n_heads * head_dim, wkv = (long)n_kv_heads * head_dim;
  if (ld_qkv < wq + 2 * wkv || ld_q < wq || ld_cache < wkv) return fail(TBP_EINVAL, "leading dimensions must cover the head columns");
  if (batch == 0 || n_new == 0) return TBP_OK;
  if (!lengths || !qkv || !q_out || !cache_k || !cache_v) return fail(TBP_EINVAL, "null pointer");
  const size_t e = dtype == TBP_BF16 ? 2 : 4;
  if (misaligned(qkv, e) || misaligned(q_out, e) || misaligned(cache_k, e) || misaligned(cache_v, e))
    return fail(TBP_EINVAL, "tensors must be aligned to their elements");
  tbp::RotaryParams p{};
  p.x = qkv; p.ld_x = ld_qkv; p.y = q_out; p.ld_y = ld_q; p.table = static_cast<const float2*>(table); p.n_pos = n_pos; p.seq = 1;
  p.rows = batch * n_new; p.heads = n_heads + 2 * n_kv_heads; p.dh = head_dim; p.half = rot_dim / 2; p.interleaved = layout; p.sgn = 1.f;
  p.lengths = lengths; p.tokens_new = n_new; p.q_heads = n_heads; p.kv_heads = n_kv_heads;
  p.cache_k = cache_k; p.cache_v = cache_v; p.ld_c = ld_cache; p.capacity = capacity; p.sinks = sinks;
  TBP_HIP(tbp::rotary_append(dtype, p, stream_of(stream)));
  return TBP_OK;
}

// ---- log probabilities -------------------------------------------------------------------------------------------------------
static tbp_status check_logits(int dtype, int rows, int vocab, const void* logits, int64_t ld) {
  if (check_storage(dtype) != TBP_OK) return TBP_EINVAL;
  if (rows < 0 || vocab < 1) return fail(TBP_EINVAL, "rows must be at least 0 and vocab at least 1");
  if (vocab > (1 << 24)) return fail(TBP_EINVAL, "vocab %d above the limit %d", vocab, 1 << 24);
  if (ld < vocab) return fail(TBP_EINVAL, "leading dimension smaller than vocab");
  if (rows && (!logits || misaligned(logits, dtype == TBP_BF16 ? 2 : 4))) return fail(TBP_EINVAL, "logits must be non-null and aligned to their elements");
  return TBP_OK;
}

tbp_status tbp_logprobs(int dtype, int rows, int vocab, const void* logits, int64_t ld_logits, const int32_t* targets, float* logp,
                        float* entropy, float* lse, int top, float* top_logp, int32_t* top_ids, void* stream) {
  if (check_logits(dtype, rows, vocab, logits, ld_logits) != TBP_OK) return TBP_EINVAL;
  if (top < 0 || top > tbp::kMaxTop || top > vocab) return fail(TBP_EINVAL, "top must be 0 .. %d and at most vocab", tbp::kMaxTop);
  if (rows == 0) return TBP_OK;
  if (!targets || !logp || !entropy || !lse || (top && (!top_logp || !top_ids))) return fail(TBP_EINVAL, "null pointer");
  tbp::LogprobParams p{};
  p.logits = logits; p.ld = ld_logits; p.rows = rows; p.vocab = vocab; p.targets = targets; p.logp = logp; p.entropy = entropy; p.lse = lse;
  p.top = top; p.top_logp = top_logp; p.top_ids = top_ids;
  TBP_HIP(tbp::logprobs(dtype, p, stream_of(stream)));
  return TBP_OK;
}

tbp_status tbp_logprobs_p1(int dtype, int rows, int vocab, const void* logits, int64_t ld_logits, const int32_t* targets,
                           const float* lse, const float* entropy, const float* d_logp, const float* d_entropy, void* d_logits,
                           int64_t ld_d, void* stream) {
  if (check_logits(dtype, rows, vocab, logits, ld_logits) != TBP_OK) return TBP_EINVAL;
  if (ld_d < vocab) return fail(TBP_EINVAL, "leading dimension smaller than vocab");
  if (rows == 0) return TBP_OK;
  if (!targets || !lse || !entropy || !d_logp || !d_logits) return fail(TBP_EINVAL, "null pointer");
  if (misaligned(d_logits, dtype == TBP_BF16 ? 2 : 4)) return fail(TBP_EINVAL, "d_logits must be aligned to its elements");
  if (d_logits == logits && ld_d != ld_logits) return fail(TBP_EINVAL, "in place both leading dimensions must be the same");
  tbp::LogprobParams p{};
  p.logits = logits; p.ld = ld_logits; p.rows = rows; p.vocab = vocab; p.targets = targets;
  p.lse = const_cast<float*>(lse); p.entropy = const_cast<float*>(entropy); p.d_logp = d_logp; p.d_entropy = d_entropy;
  p.d_logits = d_logits; p.ld_d = ld_d;
  TBP_HIP(tbp::logprobs_p1(dtype, p, stream_of(stream)));
  return TBP_OK;
}

tbp_status tbp_logprobs_step(int dtype, int rows, int vocab, const void* logits, int64_t ld_logits, const int32_t* targets,
                             const float* d_logp, const float* d_entropy, float* logp, float* entropy, float* lse, void* d_logits,
                             int64_t ld_d, void* stream) {
  if (check_logits(dtype, rows, vocab, logits, ld_logits) != TBP_OK) return TBP_EINVAL;
  if (ld_d < vocab) return fail(TBP_EINVAL, "leading dimension smaller than vocab");
  if (rows == 0) return TBP_OK;
  if (!targets || !lse || !entropy || !logp || !d_logp || !d_logits) return fail(TBP_EINVAL, "null pointer");
  if (misaligned(d_logits, dtype == TBP_BF16 ? 2 : 4)) return fail(TBP_EINVAL, "d_logits must be aligned to its elements");
  if (d_logits == logits && ld_d != ld_logits) return fail(TBP_EINVAL, "in place both leading dimensions must be the same");
  tbp::LogprobParams p{};
  p.logits = logits; p.ld = ld_logits; p.rows = rows; p.vocab = vocab; p.targets = targets; p.logp = logp; p.entropy = entropy; p.lse = lse;
  p.d_logp = d_logp; p.d_entropy = d_entropy; p.d_logits = d_logits; p.ld_d = ld_d;
  TBP_HIP(tbp::logprobs_step(dtype, p, stream_of(stream)));
  return TBP_OK;
}

// ---- the norm over gradient tensors, and clipping ----------------------------------------------------------------------------
size_t tbp_grad_workspace_bytes(int n) {
  const size_t tables = n > 0 ? ((size_t)n + tbp::kGradTable - 1) / tbp::kGradTable : 1;
  return tables * tbp::kGradSums * sizeof(double);
}

static tbp_status check_grads(int dtype, int n, const void* const* grads, const int64_t* counts, const void* workspace) {
  if (check_storage(dtype) != TBP_OK) return TBP_EINVAL;
  if (n < 0 || n > (1 << 20)) return fail(TBP_EINVAL, "the number of tensors must be 0 .. %d", 1 << 20);
  if (n && (!grads || !counts)) return fail(TBP_EINVAL, "null pointer");
  if (!workspace || misaligned(workspace, 256)) return fail(TBP_EINVAL, "workspace must be non-null and 256-byte aligned");
  for (int i = 0; i < n; i++) {
    if (counts[i] < 0 || counts[i] > ((int64_t)1 << 42)) return fail(TBP_EINVAL, "tensor %d: bad element count", i);
    if (counts[i] && (!grads[i] || misaligned(grads[i], dtype == TBP_BF16 ? 2 : 4)))
      return fail(TBP_EINVAL, "tensor %d must be non-null and aligned to its elements", i);
  }
  return TBP_OK;
}

tbp_status tbp_grad_sumsq(int dtype, int n, const void* const* grads, const int64_t* counts, double* sumsq, void* workspace,
                          void* stream) {
  if (check_grads(dtype, n, grads, counts, workspace) != TBP_OK) return TBP_EINVAL;
  if (!sumsq || misaligned(sumsq, 8)) return fail(TBP_EINVAL, "sumsq must be non-null and 8-byte aligned");
  int n_sums = 0;
  double* const sums = static_cast<double*>(workspace);
  TBP_HIP(tbp::grad_sumsq(dtype, n, grads, counts, sums, &n_sums, stream_of(stream)));
  TBP_HIP(tbp::grad_sum(sums, n_sums, sumsq, stream_of(stream)));
  return TBP_OK;
}

tbp_status tbp_grad_clip(int dtype, int out_dtype, int n, const void* const* grads, void* const* outs, const int64_t* counts,
                         const double* sumsq, float max_norm, float* norm, void* workspace, void* stream) {
  if (check_grads(dtype, n, grads, counts, workspace) != TBP_OK || check_storage(out_dtype) != TBP_OK) return TBP_EINVAL;
  if (!(max_norm >= 0.f)) return fail(TBP_EINVAL, "max_norm must be at least 0");
  if (n && !outs) return fail(TBP_EINVAL, "null pointer");
  if (sumsq && misaligned(sumsq, 8)) return fail(TBP_EINVAL, "sumsq must be 8-byte aligned");
  for (int i = 0; i < n; i++) {
    if (counts[i] && (!outs[i] || misaligned(outs[i], out_dtype == TBP_BF16 ? 2 : 4)))
      return fail(TBP_EINVAL, "output %d must be non-null and aligned to its elements", i);
    if (counts[i] && outs[i] == grads[i] && dtype != out_dtype) return fail(TBP_EINVAL, "output %d is its gradient but has another type", i);
  }
  int n_sums = 1;
  double* const sums = static_cast<double*>(workspace);
  if (!sumsq) TBP_HIP(tbp::grad_sumsq(dtype, n, grads, counts, sums, &n_sums, stream_of(stream)));
  TBP_HIP(tbp::grad_clip(dtype, out_dtype, n, grads, outs, counts, sumsq ? sumsq : sums, n_sums, max_norm, norm, stream_of(stream)));
  return TBP_OK;
}

// ---- norms of query and key heads with rotary positions ------------------------------------------------------------------------
static tbp_status check_qk_norm(int dtype, int n_heads, int n_kv_heads, int head_dim, float eps, const void* gq, const void* gk, int rot_dim,
                                int layout, const void* table, int n_pos) {
  if (check_storage(dtype) != TBP_OK) return TBP_EINVAL;
  if (n_heads < 0 || n_kv_heads < 0) return fail(TBP_EINVAL, "negative size");
  if (head_dim < 2 || head_dim % 2 || head_dim > tbp::kQkNormMaxHead) return fail(TBP_EINVAL, "head_dim must be even and 2 .. %d", tbp::kQkNormMaxHead);
  if (((long)n_heads + 2L * n_kv_heads) * head_dim >= (1L << 30)) return fail(TBP_EINVAL, "heads too many");
  if (!(eps >= 0.f)) return fail(TBP_EINVAL, "eps must be at least 0");
  if (rot_dim && check_rotary(dtype, head_dim, rot_dim, layout, table, n_pos) != TBP_OK) return TBP_EINVAL;
  const size_t e = dtype == TBP_BF16 ? 2 : 4;
  if ((n_heads && (!gq || misaligned(gq, e))) || (n_kv_heads && (!gk || misaligned(gk, e))))
    return fail(TBP_EINVAL, "gains must be non-null and aligned to their elements");
  return TBP_OK;
}

static tbp::QkNormParams qk_norm_params(int rows, int n_heads, int n_kv_heads, int head_dim, float eps, const void* gq, const void* gk, int rot_dim,
                                        int layout, const void* table, int n_pos, const int32_t* positions, int seq) {
  tbp::QkNormParams p{};
  p.rows = rows; p.q_heads = n_heads; p.kv_heads = n_kv_heads; p.dh = head_dim; p.eps = eps; p.gq = gq; p.gk = gk;
  p.half = rot_dim / 2; p.interleaved = rot_dim ? layout : 0; p.table = static_cast<const float2*>(table); p.n_pos = n_pos;
  p.positions = positions; p.seq = seq < 1 ? 1 : seq;
  return p;
}

tbp_status tbp_qk_norm(int dtype, int rows, int n_heads, int n_kv_heads, int head_dim, float eps, const void* gq, const void* gk,
                       int rot_dim, int layout, const void* table, int n_pos, const int32_t* positions, int seq, const void* x,
                       int ld_x, void* y, int ld_y, void* stream) {
  if (rows < 0) return fail(TBP_EINVAL, "negative size");
  if (check_qk_norm(dtype, n_heads, n_kv_heads, head_dim, eps, gq, gk, rot_dim, layout, table, n_pos) != TBP_OK) return TBP_EINVAL;
  if (rot_dim && !positions && seq < 1) return fail(TBP_EINVAL, "without positions seq must be at least 1");
  const long columns = ((long)n_heads + n_kv_heads) * head_dim;
  if (ld_x < columns || ld_y < columns) return fail(TBP_EINVAL, "leading dimensions must cover the %ld head columns", columns);
  if (rows == 0 || columns == 0) return TBP_OK;
  if (!x || !y) return fail(TBP_EINVAL, "null pointer");
  const size_t e = dtype == TBP_BF16 ? 2 : 4;
  if (misaligned(x, e) || misaligned(y, e)) return fail(TBP_EINVAL, "tensors must be aligned to their elements");
  if (x == y && ld_x != ld_y) return fail(TBP_EINVAL, "in place both leading dimensions must be the same");
  tbp::QkNormParams p = qk_norm_params(rows, n_heads, n_kv_heads, head_dim, eps, gq, gk, rot_dim, layout, table, n_pos, positions, seq);
  p.x = x; p.ld_x = ld_x; p.y = y; p.ld_y = ld_y;
  TBP_HIP(tbp::qk_norm(dtype, p, stream_of(stream)));
  return TBP_OK;
}

int tbp_qk_norm_heads_per_thread(int dtype, int rows, int n_heads, int n_kv_heads, int head_dim) {
  if (check_storage(dtype) != TBP_OK || rows < 0 || n_heads < 0 || n_kv_heads < 0 || head_dim < 2 || head_dim > tbp::kQkNormMaxHead ||
      ((long)n_heads + 2L * n_kv_heads) * head_dim >= (1L << 30)) return 0;      // (no such call)
  return tbp::qk_norm_heads_per_thread(dtype, rows, n_heads, n_kv_heads, head_dim);
}

int tbp_qk_norm_partial_rows(int rows, int n_heads, int n_kv_heads, int head_dim) {
  if (rows < 1 || n_heads < 0 || n_kv_heads < 0 || n_heads + (long)n_kv_heads < 1 || head_dim < 2) return 0;
  return tbp::qk_norm_partial_rows(rows, n_heads, n_kv_heads, head_dim);
}

tbp_status tbp_qk_norm_p1(int dtype, int rows, int n_heads, int n_kv_heads, int head_dim, float eps, const void* gq, const void* gk,
                          int rot_dim, int layout, const void* table, int n_pos, const int32_t* positions, int seq, const void* dy,
                          int ld_dy, const void* x, int ld_x, void* dx, int ld_dx, float* partials_out, void* stream) {
  if (rows < 0) return fail(TBP_EINVAL, "negative size");
  if (check_qk_norm(dtype, n_heads, n_kv_heads, head_dim, eps, gq, gk, rot_dim, layout, table, n_pos) != TBP_OK) return TBP_EINVAL;
  if (rot_dim && !positions && seq < 1) return fail(TBP_EINVAL, "without positions seq must be at least 1");
  const long columns = ((long)n_heads + n_kv_heads) * head_dim;
  if (ld_x < columns || ld_dy < columns || ld_dx < columns) return fail(TBP_EINVAL, "leading dimensions must cover the %ld head columns", columns);
  if (rows == 0 || columns == 0) return TBP_OK;
  if (!dy || !x || !dx || !partials_out) return fail(TBP_EINVAL, "null pointer");
  const size_t e = dtype == TBP_BF16 ? 2 : 4;
  if (misaligned(dy, e) || misaligned(x, e) || misaligned(dx, e) || misaligned(partials_out, 4)) return fail(TBP_EINVAL, "tensors must be aligned to their elements");
  if (dx == dy && ld_dx != ld_dy) return fail(TBP_EINVAL, "in place both leading dimensions must be the same");
  if (dx == x) return fail(TBP_EINVAL, "dx may be dy, not x");
  tbp::QkNormParams p = qk_norm_params(rows, n_heads, n_kv_heads, head_dim, eps, gq, gk, rot_dim, layout, table, n_pos, positions, seq);
  p.x = x; p.ld_x = ld_x; p.dy = dy; p.ld_dy = ld_dy; p.y = dx; p.ld_y = ld_dx; p.partials = partials_out;
  TBP_HIP(tbp::qk_norm_p1(dtype, p, stream_of(stream)));
  return TBP_OK;
}

tbp_status tbp_qk_norm_append(int dtype, int batch, int n_new, int n_heads, int n_kv_heads, int head_dim, float eps, const void* gq,
                              const void* gk, int rot_dim, int layout, const void* table, int n_pos, const int32_t* lengths,
                              const void* qkv, int ld_qkv, void* q_out, int ld_q, void* cache_k, void* cache_v, int ld_cache,
                              int capacity, int sinks, void* stream) {
  if (check_heads(n_heads, n_kv_heads, head_dim) != TBP_OK) return TBP_EINVAL;
  if (check_qk_norm(dtype, n_heads, n_kv_heads, head_dim, eps, gq, gk, rot_dim, layout, table, n_pos) != TBP_OK) return TBP_EINVAL;
  if (batch < 0 || n_new < 0) return fail(TBP_EINVAL, "negative size");
  if ((long)batch * n_new > 0x7fffffffL) return fail(TBP_EINVAL, "batch * n_new too large");
  if (sinks < 0 || capacity <= sinks) return fail(TBP_EINVAL, "capacity must be above sinks, sinks at least 0");
  const long wq = (long)n_heads * head_dim, wkv = (long)n_kv_heads * head_dim;
  if (ld_qkv < wq + 2 * wkv || ld_q < wq || ld_cache < wkv) return fail(TBP_EINVAL, "leading dimensions must cover the head columns");
  if (batch == 0 || n_new == 0) return TBP_OK;
  if (!lengths || !qkv || !q_out || !cache_k || !cache_v) return fail(TBP_EINVAL, "null pointer");
  const size_t e = dtype == TBP_BF16 ? 2 : 4;
  if (misaligned(qkv, e) || misaligned(q_out, e) || misaligned(cache_k, e) || misaligned(cache_v, e))
    return fail(TBP_EINVAL, "tensors must be aligned to their elements");
  tbp::QkNormParams p = qk_norm_params(batch * n_new, n_heads, n_kv_heads, head_dim, eps, gq, gk, rot_dim, layout, table, n_pos, nullptr, 1);
  p.x = qkv; p.ld_x = ld_qkv; p.y = q_out; p.ld_y = ld_q; p.lengths = lengths; p.tokens_new = n_new;
  p.cache_k = cache_k; p.cache_v = cache_v; p.ld_c = ld_cache; p.capacity = capacity; p.sinks = sinks;
  TBP_HIP(tbp::qk_norm_append(dtype, p, stream_of(stream)));
  return TBP_OK;
}

// ---- causal attention over packed sequences ------------------------------------------------------------------------------------
static tbp_status check_packed(int dtype, int n_seqs, int rows, int n_heads, int n_kv_heads, int head_dim) {
  if (dtype != TBP_BF16) return fail(TBP_EINVAL, "packed attention is built for bf16 storage only");
  if (head_dim != 64 && head_dim != 128) return fail(TBP_EINVAL, "packed attention needs head_dim 64 or 128");
  if (check_heads(n_heads, n_kv_heads, head_dim) != TBP_OK) return TBP_EINVAL;
  if (n_seqs < 0 || rows < 0) return fail(TBP_EINVAL, "negative size");
  if (rows > (1 << 22) || n_seqs > (1 << 20)) return fail(TBP_EINVAL, "rows above 2^22 or n_seqs above 2^20");
  if ((long)n_heads * (rows / 32 + n_seqs + 1) >= (1L << 23)) return fail(TBP_EINVAL, "n_heads * (rows / 32 + n_seqs + 1) must be below 2^23");      // (threads of a launch are counted in 32 bits)
  return TBP_OK;
}

tbp_status tbp_packed_attention_fwd(int dtype, int n_seqs, int rows, int n_heads, int n_kv_heads, int head_dim, const int32_t* starts,
                                    const void* qkv, int ld_qkv, void* out, int ld_out, float* lse, void* stream) {
  if (check_packed(dtype, n_seqs, rows, n_heads, n_kv_heads, head_dim) != TBP_OK) return TBP_EINVAL;
  if (rows == 0) return TBP_OK;
  if (!starts || !qkv || !out || !lse) return fail(TBP_EINVAL, "null pointer");
  if (check_ld("ld_qkv", ld_qkv, ((long)n_heads + 2L * n_kv_heads) * head_dim) != TBP_OK) return TBP_EINVAL;
  if (check_ld("ld_out", ld_out, (long)n_heads * head_dim) != TBP_OK) return TBP_EINVAL;
  if (misaligned(qkv, 16) || misaligned(out, 16)) return fail(TBP_EINVAL, "qkv and out must be 16-byte aligned");
  TBP_HIP(tbp::packed_attention_fwd(tbp::PackedShape{starts, n_seqs, rows, n_heads, n_kv_heads, head_dim}, qkv, ld_qkv, out, ld_out, lse, stream_of(stream)));
  return TBP_OK;
}

tbp_status tbp_packed_attention_plan(int n_seqs, int rows, int n_heads, int n_kv_heads, int head_dim, tbp_packed_plan* plan) {
  if (!plan) return fail(TBP_EINVAL, "plan must be non-null");
  if (check_packed(TBP_BF16, n_seqs, rows, n_heads, n_kv_heads, head_dim) != TBP_OK) return TBP_EINVAL;
  const tbp::PackedPlan p = tbp::packed_plan(tbp::PackedShape{nullptr, n_seqs, rows, n_heads, n_kv_heads, head_dim});
  *plan = tbp_packed_plan{p.query_heads, p.key_shares, p.scores_ahead, p.queries_most_first, p.keys, p.parts, p.keys_most_first};
  return TBP_OK;
}

size_t tbp_packed_attention_p1_scratch_bytes(int n_seqs, int rows, int n_heads, int n_kv_heads, int head_dim) {
  if (rows < 1 || check_packed(TBP_BF16, n_seqs, rows, n_heads, n_kv_heads, head_dim) != TBP_OK) return 0;
  return delta_bytes(1, n_heads, rows) + tbp::packed_attention_p1_partial_bytes(tbp::PackedShape{nullptr, n_seqs, rows, n_heads, n_kv_heads, head_dim});
}

tbp_status tbp_packed_attention_p1(int dtype, int n_seqs, int rows, int n_heads, int n_kv_heads, int head_dim, const int32_t* starts,
                                   const void* qkv, int ld_qkv, const void* out, const void* d_out, int ld_out, const float* lse,
                                   void* dqkv, int ld_dqkv, void* scratch, void* stream) {
  if (check_packed(dtype, n_seqs, rows, n_heads, n_kv_heads, head_dim) != TBP_OK) return TBP_EINVAL;
  if (rows == 0) return TBP_OK;
  if (!starts || !qkv || !out || !d_out || !lse || !dqkv || !scratch) return fail(TBP_EINVAL, "null pointer");
  const long columns = ((long)n_heads + 2L * n_kv_heads) * head_dim;
  if (check_ld("ld_qkv", ld_qkv, columns) != TBP_OK || check_ld("ld_dqkv", ld_dqkv, columns) != TBP_OK) return TBP_EINVAL;
  if (check_ld("ld_out", ld_out, (long)n_heads * head_dim) != TBP_OK) return TBP_EINVAL;
  if (misaligned(qkv, 16) || misaligned(out, 16) || misaligned(d_out, 16) || misaligned(dqkv, 16) || misaligned(scratch, 256))
    return fail(TBP_EINVAL, "tensors must be 16-byte aligned, scratch 256-byte aligned");
  TBP_HIP(tbp::packed_attention_p1(tbp::PackedShape{starts, n_seqs, rows, n_heads, n_kv_heads, head_dim}, qkv, ld_qkv, out, d_out, ld_out, lse, dqkv, ld_dqkv,
                                   static_cast<float*>(scratch), reinterpret_cast<float*>(static_cast<char*>(scratch) + delta_bytes(1, n_heads, rows)),
                                   stream_of(stream)));
  return TBP_OK;
}

// ---- a stash in 8 bits -----------------------------------------------------------------------------------------------------------
static tbp_status check_stash8(int slots, int tokens, int cols) {
  if (slots < 0 || tokens < 1 || cols < 1) return fail(TBP_EINVAL, "slots must be at least 0, tokens and cols at least 1");
  if (tokens > (1 << 22) || cols >= (1 << 22)) return fail(TBP_EINVAL, "tokens above 2^22, or cols not below it");
  if ((long)slots * ((tokens + 63) / 64) >= (1L << 30)) return fail(TBP_EINVAL, "slots * tokens too large");
  return TBP_OK;
}

static size_t stash8_data_bytes(int slots, int tokens, int cols) { return (size_t)slots * ((tokens + 63) / 64) * ((cols + 31) / 32) * 2048; }

static tbp::Stash8Slot stash8_slot(int slots, int tokens, int cols, int slot, const void* stash) {
  tbp::Stash8Slot p{};
  p.data = static_cast<unsigned char*>(const_cast<void*>(stash));
  p.scales = reinterpret_cast<float*>(p.data + stash8_data_bytes(slots, tokens, cols));
  p.tokens = tokens; p.cols = cols; p.slot = slot;
  p.steps = (tokens + 63) / 64; p.blocks = (tokens + tbp::kStash8Block - 1) / tbp::kStash8Block; p.col_blocks = (cols + 31) / 32;
  return p;
}

size_t tbp_stash8_bytes(int slots, int tokens, int cols) {
  if (check_stash8(slots, tokens, cols) != TBP_OK) return 0;
  if (slots == 0) { fail(TBP_EINVAL, "a stash must have slots, at least 1"); return 0; }
  return stash8_data_bytes(slots, tokens, cols) + (size_t)slots * ((tokens + tbp::kStash8Block - 1) / tbp::kStash8Block) * ((cols + 31) / 32) * 32 * sizeof(float);
}

static tbp_status check_stash8_slot(int dtype, int slots, int tokens, int cols, int slot, const void* x, int ld, const void* stash) {
  if (check_storage(dtype) != TBP_OK || check_stash8(slots, tokens, cols) != TBP_OK) return TBP_EINVAL;
  if (slot < 0 || slot >= slots) return fail(TBP_EINVAL, "slot %d of %d", slot, slots);
  if (ld < cols) return fail(TBP_EINVAL, "leading dimension smaller than cols");
  if (!x || !stash) return fail(TBP_EINVAL, "null pointer");
  if (misaligned(x, dtype == TBP_BF16 ? 2 : 4) || misaligned(stash, 16)) return fail(TBP_EINVAL, "the tensor must be aligned to its elements, the stash to 16 bytes");
  return TBP_OK;
}

tbp_status tbp_stash8_put(int dtype, int slots, int tokens, int cols, int slot, const void* x, int ld_x, void* stash, void* stream) {
  if (check_stash8_slot(dtype, slots, tokens, cols, slot, x, ld_x, stash) != TBP_OK) return TBP_EINVAL;
  TBP_HIP(tbp::stash8_put(dtype, stash8_slot(slots, tokens, cols, slot, stash), x, ld_x, stream_of(stream)));
  return TBP_OK;
}

tbp_status tbp_stash8_get(int dtype, int slots, int tokens, int cols, int slot, const void* stash, void* y, int ld_y, void* stream) {
  if (check_stash8_slot(dtype, slots, tokens, cols, slot, y, ld_y, stash) != TBP_OK) return TBP_EINVAL;
  TBP_HIP(tbp::stash8_get(dtype, stash8_slot(slots, tokens, cols, slot, stash), y, ld_y, stream_of(stream)));
  return TBP_OK;
}

size_t tbp_stash8_dw_workspace_bytes(int tokens, int m, int n_out, int n) {
  if (n < 1 || check_stash8(n, tokens, m) != TBP_OK || check_stash8(n, tokens, n_out) != TBP_OK) return 0;
  return tbp::stash8_plan(m, n_out, n * ((tokens + 63) / 64), n * ((tokens + tbp::kStash8Block - 1) / tbp::kStash8Block)).bytes;
}

tbp_status tbp_stash8_dw_plan(int tokens, int m, int n_out, int n, int* tile, int* shares) {
  if (!tile || !shares) return fail(TBP_EINVAL, "outputs must be non-null");
  if (check_stash8(n, tokens, m) != TBP_OK || check_stash8(n, tokens, n_out) != TBP_OK) return TBP_EINVAL;
  const tbp::Stash8Plan plan = tbp::stash8_plan(m, n_out, n * ((tokens + 63) / 64), n * ((tokens + tbp::kStash8Block - 1) / tbp::kStash8Block));
  *tile = 64 * plan.mb; *shares = plan.shares;
  return TBP_OK;
}

tbp_status tbp_stash8_dw(int slots, int tokens, int m, int n_out, int first, int n, const void* x_stash, const void* dy_stash, float* dw,
                         int ld_dw, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (check_stash8(slots, tokens, m) != TBP_OK || check_stash8(slots, tokens, n_out) != TBP_OK) return TBP_EINVAL;
  if (first < 0 || n < 0 || first > slots - n) return fail(TBP_EINVAL, "slots %d .. %ld of %d", first, (long)first + n - 1, slots);
  if (ld_dw < n_out) return fail(TBP_EINVAL, "leading dimension smaller than n_out");
  if (n == 0 && accumulate) return TBP_OK;
  if (!x_stash || !dy_stash || !dw) return fail(TBP_EINVAL, "null pointer");
  if (misaligned(x_stash, 16) || misaligned(dy_stash, 16) || misaligned(dw, 4)) return fail(TBP_EINVAL, "stashes must be 16-byte aligned, dw 4-byte");
  const size_t need = tbp_stash8_dw_workspace_bytes(tokens, m, n_out, n);
  if (need && (!workspace || misaligned(workspace, 256) || workspace_bytes < need)) return fail(TBP_EINVAL, "workspace must be 256-byte aligned and have %zu bytes", need);
  TBP_HIP(tbp::stash8_dw(stash8_slot(slots, tokens, m, first, x_stash), stash8_slot(slots, tokens, n_out, first, dy_stash), n, dw, ld_dw, accumulate,
                         static_cast<float*>(workspace), stream_of(stream)));
  return TBP_OK;
}

}  // extern "C"
