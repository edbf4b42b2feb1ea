"""Binding of the operators for long contexts, the last stage and serving: sliding-window attention with sinks, rotary
positions, log probabilities of tokens, the norm of all gradients with clipping; and of those of a stage that is trained on packed
documents: norms of query and key heads, attention over packed sequences, a stash in 8 bits.

As in binding.py: argument marshalling only, on torch's current stream; outputs and workspaces are allocated where the caller
passes none.  Index tensors (lengths, positions, targets) are int32.  The checks here are those that the C entry points cannot
make (types, shapes and strides of tensors, the sizes of memory, and that all of it is on the current device); the single-token
calls are bound by the host, which is why they are written out rather than shared by many small functions.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import TBP_BF16, TBP_F32, _check, lib

__all__ = [
    "TBP_ROTARY_HALF", "TBP_ROTARY_INTERLEAVED", "TBP_ROTARY_PLAIN", "TBP_ROTARY_LINEAR", "TBP_ROTARY_BASE", "TBP_ROTARY_RAMP",
    "tbp_rotary_scale", "tbp_rotary_table", "tbp_rotary", "tbp_rotary_append", "tbp_window_attention_fwd", "tbp_window_attention_p1",
    "tbp_window_decode_workspace", "tbp_window_decode", "tbp_logprobs", "tbp_logprobs_p1", "tbp_logprobs_step", "GradList",
    "tbp_qk_norm", "tbp_qk_norm_p1", "tbp_qk_norm_append", "tbp_packed_attention_fwd", "tbp_packed_attention_p1", "tbp_packed_plan", "tbp_packed_attention_plan", "Stash8", "tbp_stash8_dw", "tbp_stash8_dw_plan",
]

TBP_ROTARY_HALF, TBP_ROTARY_INTERLEAVED = 0, 1
TBP_ROTARY_PLAIN, TBP_ROTARY_LINEAR, TBP_ROTARY_BASE, TBP_ROTARY_RAMP = 0, 1, 2, 3

_F32, _I32 = torch.float32, torch.int32
_CODE = {torch.bfloat16: TBP_BF16, torch.float32: TBP_F32}


class tbp_rotary_scale(C.Structure):
    _fields_ = [("scaling", C.c_int32), ("factor", C.c_float), ("low", C.c_float), ("high", C.c_float), ("original", C.c_float),
                ("magnitude", C.c_float)]


class tbp_packed_plan(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("query_heads", "key_shares", "scores_ahead", "queries_most_first", "keys", "parts", "keys_most_first")]


def _dt(t):
    try:
        return _CODE[t.dtype]
    except KeyError:
        raise TypeError(f"unsupported tensor dtype {t.dtype}") from None


def _stream_of(device, *others):
    """torch's current stream, which is that of the current device: `device`, a tensor's get_device().  The others that the caller has brought (None: none)
    have to be there too."""
    for t in others:
        if t is not None and t.get_device() != device:
            raise TypeError(f"tensors of one call must be on one GPU, not on {t.device} and {f'cuda:{device}' if device >= 0 else 'the host'}")
    if device < 0:
        raise TypeError("tensors must be on the GPU")
    if device != torch._C._cuda_getDevice():
        raise TypeError(f"tensors are on the GPU cuda:{device}, which is not the current one")
    return torch._C._cuda_getCurrentRawStream(device)


def _vector(t, n, dtype, what):
    """The address of a contiguous vector of n entries (None: null)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{what} must be a contiguous {dtype} tensor of {n} entries")
    return t.data_ptr()


def _memory(t, what):
    """(address, bytes) of a contiguous tensor that serves as plain memory (None: null)."""
    if t is None:
        return None, 0
    if not t.is_contiguous():
        raise TypeError(f"{what} must be contiguous")
    return t.data_ptr(), t.nbytes


def _matrix(t, dtype, what, rows, columns):
    """The leading dimension of a matrix of contiguous rows, of which a call reads or writes the first `rows` and of these the first `columns`."""
    if t.dtype is not dtype or t.dim() != 2:
        raise TypeError(f"{what} must be a matrix of type {dtype}")
    have, wide = t.shape
    if have < rows or wide < columns:
        raise TypeError(f"{what} must have {rows} rows of {columns} columns, not {have} of {wide}")
    ld, step = t.stride()
    if step != 1 and wide > 1:
        raise TypeError(f"{what} must have contiguous rows")
    return ld if have > 1 or ld > wide else wide


def _caches(k, v, dtype, batch, width):
    """(capacity, distance of rows) of a pair of caches."""
    shape, stride = k.shape, k.stride()
    if len(shape) != 3 or shape[0] != batch or shape[2] != width or stride[2] != 1 or (batch > 1 and stride[0] != shape[1] * stride[1]):
        raise TypeError("caches must be [batch, capacity, n_kv_heads*head_dim] with contiguous rows of one distance")
    if v.shape != shape or v.stride() != stride or k.dtype is not dtype or v.dtype is not dtype:
        raise TypeError("both caches must have one shape, one stride, and the tokens' type")
    return shape[1], stride[1]


def _sequences(rows, seq):
    if seq < 1 or rows % seq:
        raise ValueError(f"{rows} rows are no whole sequences of {seq}")
    return rows // seq


# ---- sliding-window attention ------------------------------------------------------------------------------------------
def tbp_window_attention_fwd(qkv, seq, n_heads, n_kv_heads, head_dim, window, sinks=0, lengths=None, out=None, lse=None):
    """qkv [batch*seq, (n_heads + 2 n_kv_heads) head_dim] (q | k | v, rotated) -> (out [batch*seq, n_heads*head_dim], lse2 [batch, heads, seq])."""
    rows, dt = qkv.shape[0], qkv.dtype
    batch, ld_out = _sequences(rows, seq), n_heads * head_dim
    ld_qkv = _matrix(qkv, dt, "qkv", rows, (n_heads + 2 * n_kv_heads) * head_dim)
    given = out, lse
    if out is None:
        out = qkv.new_empty((rows, ld_out))
    else:
        ld_out = _matrix(out, dt, "out", rows, ld_out)
    if lse is None:
        lse = qkv.new_empty((batch, n_heads, seq), dtype=_F32)
    else:
        _vector(lse, batch * n_heads * seq, _F32, "lse")
    _check(lib().tbp_window_attention_fwd(_dt(qkv), batch, n_heads, n_kv_heads, seq, head_dim, window, sinks, _vector(lengths, batch, _I32, "lengths"),
                                          qkv.data_ptr(), ld_qkv, out.data_ptr(), ld_out, lse.data_ptr(), _stream_of(qkv.get_device(), lengths, *given)))
    return out, lse


def tbp_window_attention_p1(qkv, out, d_out, lse, seq, n_heads, n_kv_heads, head_dim, window, sinks=0, lengths=None, dqkv=None, scratch=None):
    """-> dqkv [batch*seq, (n_heads + 2 n_kv_heads) head_dim] (dq | dk | dv, not rotated back)."""
    rows, dt = qkv.shape[0], qkv.dtype
    batch, ld_dqkv = _sequences(rows, seq), (n_heads + 2 * n_kv_heads) * head_dim
    ld_qkv, ld_out = _matrix(qkv, dt, "qkv", rows, ld_dqkv), _matrix(out, dt, "out", rows, n_heads * head_dim)
    if d_out.shape != out.shape or _matrix(d_out, dt, "d_out", rows, n_heads * head_dim) != ld_out:
        raise TypeError("d_out must have out's shape and leading dimension")
    given = dqkv, scratch
    if dqkv is None:
        dqkv = qkv.new_empty((rows, ld_dqkv))
    else:
        ld_dqkv = _matrix(dqkv, dt, "dqkv", rows, ld_dqkv)
    L = lib()
    need = L.tbp_window_attention_p1_scratch_bytes(batch, n_heads, n_kv_heads, seq, head_dim, window, sinks)
    if scratch is None:
        scratch = qkv.new_empty(need, dtype=torch.uint8)
    at, nbytes = _memory(scratch, "scratch")
    if nbytes < need:
        raise ValueError(f"scratch must have {need} bytes, not {nbytes}")
    _check(L.tbp_window_attention_p1(_dt(qkv), batch, n_heads, n_kv_heads, seq, head_dim, window, sinks, _vector(lengths, batch, _I32, "lengths"),
                                     qkv.data_ptr(), ld_qkv, out.data_ptr(), d_out.data_ptr(), ld_out,
                                     _vector(lse, batch * n_heads * seq, _F32, "lse"), dqkv.data_ptr(), ld_dqkv,
                                     at, _stream_of(qkv.get_device(), lengths, out, d_out, lse, *given)))
    return dqkv


def tbp_window_decode_workspace(batch, n_heads, n_kv_heads, head_dim, window, sinks=0, device="cuda"):
    """The workspace of tbp_window_decode calls of these sizes (which must not overlap), or None where they need none."""
    nbytes = lib().tbp_window_decode_workspace_bytes(batch, n_heads, n_kv_heads, head_dim, window, sinks)
    return torch.zeros(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def tbp_window_decode(q, cache_k, cache_v, lengths, n_heads, n_kv_heads, head_dim, window, sinks=0, out=None, lse=None, workspace=None):
    """q [batch, n_heads*head_dim] of the token at position lengths[b] - 1 over caches [batch, capacity, n_kv_heads*head_dim] ->
    (out [batch, n_heads*head_dim], lse2 [batch, heads]).  A program that decodes keeps a workspace (tbp_window_decode_workspace)."""
    batch, dt = q.shape[0], q.dtype
    capacity, ld_cache = _caches(cache_k, cache_v, dt, batch, n_kv_heads * head_dim)
    ld_out = n_heads * head_dim
    ld_q = _matrix(q, dt, "q", batch, ld_out)
    given = out, lse, workspace
    if out is None:
        out = q.new_empty((batch, ld_out))
    else:
        ld_out = _matrix(out, dt, "out", batch, ld_out)
    if lse is None:
        lse = q.new_empty((batch, n_heads), dtype=_F32)
    else:
        _vector(lse, batch * n_heads, _F32, "lse")
    if workspace is None:
        workspace = tbp_window_decode_workspace(batch, n_heads, n_kv_heads, head_dim, window, sinks, q.device)
    at, nbytes = _memory(workspace, "workspace")
    _check(lib().tbp_window_decode(_dt(q), batch, n_heads, n_kv_heads, head_dim, window, sinks, capacity, _vector(lengths, batch, _I32, "lengths"),
                                   q.data_ptr(), ld_q, cache_k.data_ptr(), cache_v.data_ptr(), ld_cache, out.data_ptr(),
                                   ld_out, lse.data_ptr(), at, nbytes, _stream_of(q.get_device(), cache_k, cache_v, lengths, *given)))
    return out, lse


# ---- rotary positions ----------------------------------------------------------------------------------------------------
def tbp_rotary_table(n_pos, rot_dim, base, scaling=TBP_ROTARY_PLAIN, factor=1.0, low=1.0, high=32.0, original=4096.0, magnitude=1.0,
                     device="cuda"):
    """-> table [n_pos, rot_dim/2, 2] of cosines and sines."""
    t = torch.empty((n_pos, rot_dim // 2, 2), dtype=_F32, device=device)
    sc = tbp_rotary_scale(scaling, factor, low, high, original, magnitude)
    with torch.cuda.device(t.device):
        _check(lib().tbp_rotary_table(n_pos, rot_dim, base, C.byref(sc), t.data_ptr(), _stream_of(t.get_device())))
    return t


def _table(table):
    shape = table.shape
    if table.dtype is not _F32 or len(shape) != 3 or shape[2] != 2 or not table.is_contiguous():
        raise TypeError("the table must be a contiguous float32 tensor [n_pos, rot_dim/2, 2]")
    return shape[0], 2 * shape[1]


def tbp_rotary(x, n_heads, head_dim, table, positions=None, seq=None, layout=TBP_ROTARY_HALF, backward=False, out=None):
    """The first n_heads*head_dim columns of x [rows, ld], turned (backward: the derivative).  seq: tokens per sequence, where no positions
    are given (None: all rows are one sequence).  out: new [rows, n_heads*head_dim], or the tensor to write to (x itself: in place)."""
    n_pos, rot_dim = _table(table)
    rows, dt = x.shape[0], x.dtype
    if positions is not None:
        seq = 1
    elif seq is None:
        seq = max(rows, 1)
        if rows > n_pos:
            raise ValueError(f"{rows} rows and a table of {n_pos} positions: positions or seq must be given")
    elif seq < 1:
        raise ValueError(f"seq must be at least 1, not {seq}")
    ld_out = n_heads * head_dim
    ld_x = _matrix(x, dt, "x", rows, ld_out)
    given = out
    if out is None:
        out = x.new_empty((rows, ld_out))
    else:
        ld_out = _matrix(out, dt, "out", rows, ld_out)
    _check(lib().tbp_rotary(_dt(x), rows, n_heads, head_dim, rot_dim, layout, table.data_ptr(), n_pos, _vector(positions, rows, _I32, "positions"),
                            seq, 1 if backward else 0, x.data_ptr(), ld_x, out.data_ptr(),
                            ld_out, _stream_of(x.get_device(), table, positions, given)))
    return out


def tbp_rotary_append(qkv, n_heads, n_kv_heads, head_dim, table, lengths, cache_k, cache_v, sinks=0, layout=TBP_ROTARY_HALF, q_out=None):
    """New tokens qkv [batch*n_new, (n_heads + 2 n_kv_heads) head_dim], the last ones of sequences of `lengths`: k (rotated) and v into the
    caches [batch, capacity, n_kv_heads*head_dim]; -> q rotated [batch*n_new, n_heads*head_dim]."""
    n_pos, rot_dim = _table(table)
    batch, rows, dt = lengths.shape[0], qkv.shape[0], qkv.dtype
    n_new = 0 if batch == 0 else rows // batch
    if n_new * batch != rows:
        raise ValueError(f"{rows} rows are no whole number of tokens for {batch} sequences")
    capacity, ld_cache = _caches(cache_k, cache_v, dt, batch, n_kv_heads * head_dim)
    ld_q = n_heads * head_dim
    ld_qkv = _matrix(qkv, dt, "qkv", rows, ld_q + 2 * n_kv_heads * head_dim)
    given = q_out
    if q_out is None:
        q_out = qkv.new_empty((rows, ld_q))
    else:
        ld_q = _matrix(q_out, dt, "q_out", rows, ld_q)
    _check(lib().tbp_rotary_append(_dt(qkv), batch, n_new, n_heads, n_kv_heads, head_dim, rot_dim, layout, table.data_ptr(), n_pos,
                                   _vector(lengths, batch, _I32, "lengths"), qkv.data_ptr(), ld_qkv, q_out.data_ptr(),
                                   ld_q, cache_k.data_ptr(), cache_v.data_ptr(), ld_cache, capacity, sinks, _stream_of(qkv.get_device(), table, lengths, cache_k, cache_v, given)))
    return q_out


# ---- log probabilities -----------------------------------------------------------------------------------------------------
def tbp_logprobs(logits, targets, top=0):
    """logits [rows, vocab], targets [rows] (int32; outside the vocabulary: left out) -> (logp, entropy, lse), each [rows] fp32, and with top > 0
    (top_logp [rows, top] fp32, top_ids [rows, top] int32) behind them."""
    rows, vocab = logits.shape
    stats = logits.new_empty((3, rows), dtype=_F32)
    at = stats.data_ptr()
    top_logp = top_ids = None
    if top > 0:
        top_logp = logits.new_empty((rows, top), dtype=_F32)
        top_ids = logits.new_empty((rows, top), dtype=_I32)
    _check(lib().tbp_logprobs(_dt(logits), rows, vocab, logits.data_ptr(), _matrix(logits, logits.dtype, "logits", rows, vocab), _vector(targets, rows, _I32, "targets"),
                              at, at + 4 * rows, at + 8 * rows, top, None if top_logp is None else top_logp.data_ptr(),
                              None if top_ids is None else top_ids.data_ptr(), _stream_of(logits.get_device(), targets)))
    logp, entropy, lse = stats.unbind()
    return (logp, entropy, lse, top_logp, top_ids) if top > 0 else (logp, entropy, lse)


def tbp_logprobs_p1(logits, targets, lse, entropy, d_logp, d_entropy=None, out=None):
    """-> the derivative of the logits [rows, vocab] (out: the tensor to write to, logits itself allowed)."""
    (rows, vocab), dt = logits.shape, logits.dtype
    ld_out = vocab
    given = out
    if out is None:
        out = logits.new_empty((rows, vocab))
    else:
        ld_out = _matrix(out, dt, "out", rows, vocab)
    _check(lib().tbp_logprobs_p1(_dt(logits), rows, vocab, logits.data_ptr(), _matrix(logits, dt, "logits", rows, vocab), _vector(targets, rows, _I32, "targets"),
                                 _vector(lse, rows, _F32, "lse"), _vector(entropy, rows, _F32, "entropy"), _vector(d_logp, rows, _F32, "d_logp"),
                                 _vector(d_entropy, rows, _F32, "d_entropy"), out.data_ptr(), ld_out, _stream_of(logits.get_device(), targets, lse, entropy, d_logp, d_entropy, given)))
    return out


def tbp_logprobs_step(logits, targets, d_logp, d_entropy=None, out=None):
    """Forward and derivative in one pass -> (logp, entropy, lse, d_logits)."""
    (rows, vocab), dt = logits.shape, logits.dtype
    stats = logits.new_empty((3, rows), dtype=_F32)
    at = stats.data_ptr()
    ld_out = vocab
    given = out
    if out is None:
        out = logits.new_empty((rows, vocab))
    else:
        ld_out = _matrix(out, dt, "out", rows, vocab)
    _check(lib().tbp_logprobs_step(_dt(logits), rows, vocab, logits.data_ptr(), _matrix(logits, dt, "logits", rows, vocab), _vector(targets, rows, _I32, "targets"),
                                   _vector(d_logp, rows, _F32, "d_logp"), _vector(d_entropy, rows, _F32, "d_entropy"), at, at + 4 * rows, at + 8 * rows,
                                   out.data_ptr(), ld_out, _stream_of(logits.get_device(), targets, d_logp, d_entropy, given)))
    return (*stats.unbind(), out)


# ---- the norm over gradient tensors, and clipping --------------------------------------------------------------------------
class GradList:
    """The gradient tensors of a stage (or of anything else), of one type, and where they go when they are clipped: into themselves, or
    into tensors of the same sizes and of one type.  Keeps the tensors, their addresses and a workspace; calls of one list must not overlap.
    A call raises where a tensor has been given other memory since (by an assignment to its .data, say).

    A Stage's: GradList([g for v in stage.grads.values() for g in v])."""

    def __init__(self, grads, outs=None):
        grads = list(grads)
        outs = grads if outs is None else list(outs)
        if len(outs) != len(grads) or any(o.shape != g.shape for g, o in zip(grads, outs)):
            raise ValueError("one output of the same shape is wanted for every gradient")
        if any(not t.is_contiguous() for t in grads + outs):
            raise TypeError("gradients and outputs must be contiguous")
        if len({t.dtype for t in grads}) > 1 or len({t.dtype for t in outs}) > 1 or len({t.device for t in grads + outs}) > 1:
            raise TypeError("gradients must have one type, outputs one type, and all one device")
        n, self.grads, self.outs = len(grads), grads, outs
        self._n, self._dt, self._odt = n, _dt(grads[0]) if n else 0, _dt(outs[0]) if n else 0
        self.device = grads[0].device if n else torch.device("cuda")
        self._tensors = grads if outs is grads else grads + outs
        self._at = [t.data_ptr() for t in self._tensors]
        self._src = (C.c_void_p * max(n, 1))(*self._at[:n])
        self._dst = (C.c_void_p * max(n, 1))(*self._at[-n:])
        self._counts = (C.c_int64 * max(n, 1))(*[t.numel() for t in grads])
        self._ws = torch.empty(lib().tbp_grad_workspace_bytes(n), dtype=torch.uint8, device=self.device)
        self._at_device = self._ws.get_device()

    def _in_place(self):
        if list(map(torch.Tensor.data_ptr, self._tensors)) != self._at:
            raise RuntimeError("a tensor of the list has been given other memory: make a new list")

    def sumsq(self, out=None):
        """The sum of squares [1] float64 (stages of a pipeline add theirs up before they clip)."""
        self._in_place()
        given = out
        out = torch.empty(1, dtype=torch.float64, device=self.device) if out is None else out
        _check(lib().tbp_grad_sumsq(self._dt, self._n, self._src, self._counts, _vector(out, 1, torch.float64, "out"), self._ws.data_ptr(), _stream_of(self._at_device, given)))
        return out

    def clip(self, max_norm, sumsq=None, norm=None):
        """Writes the outputs; -> the norm [1] float32.  sumsq: [1] float64, computed here where none is given."""
        self._in_place()
        given = norm
        norm = self._ws.new_empty(1, dtype=_F32) if norm is None else norm
        _check(lib().tbp_grad_clip(self._dt, self._odt, self._n, self._src, self._dst, self._counts, _vector(sumsq, 1, torch.float64, "sumsq"), max_norm,
                                   _vector(norm, 1, _F32, "norm"), self._ws.data_ptr(), _stream_of(self._at_device, sumsq, given)))
        return norm


# ---- norms of query and key heads with rotary positions ------------------------------------------------------------------------
def _norm_place(x, rows, table, positions, seq):
    """(n_pos, rot_dim, the table's address, seq) of a call on `rows` rows; no table: no rotation."""
    if table is None:
        if positions is not None:
            raise ValueError("positions without a table")
        return 0, 0, None, 1
    n_pos, rot_dim = _table(table)
    if positions is not None:
        seq = 1
    elif seq is None:
        seq = max(rows, 1)
        if rows > n_pos:
            raise ValueError(f"{rows} rows and a table of {n_pos} positions: positions or seq must be given")
    elif seq < 1:
        raise ValueError(f"seq must be at least 1, not {seq}")
    return n_pos, rot_dim, table.data_ptr(), seq


def tbp_qk_norm(qk, gq, gk, n_heads, n_kv_heads, head_dim, eps, table=None, positions=None, seq=None, layout=TBP_ROTARY_HALF, out=None):
    """The first (n_heads + n_kv_heads) head_dim columns of qk [rows, ld] (q | k), every head normed, times gq or gk [head_dim], and rotated (no table: not
    rotated).  positions, seq as for tbp_rotary.  out: new [rows, (n_heads + n_kv_heads) head_dim], or the tensor to write to (qk itself: in place)."""
    rows, dt = qk.shape[0], qk.dtype
    n_pos, rot_dim, at, seq = _norm_place(qk, rows, table, positions, seq)
    ld_out = (n_heads + n_kv_heads) * head_dim
    ld_x = _matrix(qk, dt, "qk", rows, ld_out)
    given = out
    if out is None:
        out = qk.new_empty((rows, ld_out))
    else:
        ld_out = _matrix(out, dt, "out", rows, ld_out)
    _check(lib().tbp_qk_norm(_dt(qk), rows, n_heads, n_kv_heads, head_dim, eps, _vector(gq, head_dim, dt, "gq"), _vector(gk, head_dim, dt, "gk"), rot_dim, layout,
                             at, n_pos, _vector(positions, rows, _I32, "positions"), seq, qk.data_ptr(), ld_x, out.data_ptr(), ld_out,
                             _stream_of(qk.get_device(), gq, gk, table, positions, given)))
    return out


def tbp_qk_norm_p1(d_out, qk, gq, gk, n_heads, n_kv_heads, head_dim, eps, table=None, positions=None, seq=None, layout=TBP_ROTARY_HALF, out=None, partials=None):
    """-> (dqk [rows, (n_heads + n_kv_heads) head_dim], partial rows [tbp_qk_norm_partial_rows, 2 head_dim] fp32 of the gains' gradient, for
    tbp_gain_partials_sum).  qk: the forward's input; out: the tensor to write to (d_out itself: in place); partials: rows to write them to."""
    rows, dt = qk.shape[0], qk.dtype
    n_pos, rot_dim, at, seq = _norm_place(qk, rows, table, positions, seq)
    ld_dx = (n_heads + n_kv_heads) * head_dim
    ld_x, ld_dy = _matrix(qk, dt, "qk", rows, ld_dx), _matrix(d_out, dt, "d_out", rows, ld_dx)
    given = out, partials
    if out is None:
        out = qk.new_empty((rows, ld_dx))
    else:
        ld_dx = _matrix(out, dt, "out", rows, ld_dx)
    L = lib()
    n = L.tbp_qk_norm_partial_rows(rows, n_heads, n_kv_heads, head_dim)
    if partials is None:
        partials = qk.new_empty((n, 2 * head_dim), dtype=_F32)
    else:
        _vector(partials, n * 2 * head_dim, _F32, "partials")
    _check(L.tbp_qk_norm_p1(_dt(qk), rows, n_heads, n_kv_heads, head_dim, eps, _vector(gq, head_dim, dt, "gq"), _vector(gk, head_dim, dt, "gk"), rot_dim, layout,
                            at, n_pos, _vector(positions, rows, _I32, "positions"), seq, d_out.data_ptr(), ld_dy, qk.data_ptr(), ld_x, out.data_ptr(), ld_dx,
                            partials.data_ptr(), _stream_of(qk.get_device(), d_out, gq, gk, table, positions, *given)))
    return out, partials


def tbp_qk_norm_append(qkv, gq, gk, n_heads, n_kv_heads, head_dim, eps, table, lengths, cache_k, cache_v, sinks=0, layout=TBP_ROTARY_HALF, q_out=None):
    """tbp_rotary_append with q and k normed first (table None: not rotated); -> q [batch*n_new, n_heads*head_dim]."""
    n_pos, rot_dim = (0, 0) if table is None else _table(table)
    batch, rows, dt = lengths.shape[0], qkv.shape[0], qkv.dtype
    n_new = 0 if batch == 0 else rows // batch
    if n_new * batch != rows:
        raise ValueError(f"{rows} rows are no whole number of tokens for {batch} sequences")
    capacity, ld_cache = _caches(cache_k, cache_v, dt, batch, n_kv_heads * head_dim)
    ld_q = n_heads * head_dim
    ld_qkv = _matrix(qkv, dt, "qkv", rows, ld_q + 2 * n_kv_heads * head_dim)
    given = q_out
    if q_out is None:
        q_out = qkv.new_empty((rows, ld_q))
    else:
        ld_q = _matrix(q_out, dt, "q_out", rows, ld_q)
    _check(lib().tbp_qk_norm_append(_dt(qkv), batch, n_new, n_heads, n_kv_heads, head_dim, eps, _vector(gq, head_dim, dt, "gq"), _vector(gk, head_dim, dt, "gk"),
                                    rot_dim, layout, None if table is None else table.data_ptr(), n_pos, _vector(lengths, batch, _I32, "lengths"), qkv.data_ptr(),
                                    ld_qkv, q_out.data_ptr(), ld_q, cache_k.data_ptr(), cache_v.data_ptr(), ld_cache, capacity, sinks,
                                    _stream_of(qkv.get_device(), gq, gk, table, lengths, cache_k, cache_v, given)))
    return q_out


# ---- causal attention over packed sequences ------------------------------------------------------------------------------------
def _starts(starts):
    if starts.dim() != 1 or starts.shape[0] < 1:
        raise TypeError("starts must be a vector of n_seqs + 1 entries")
    return _vector(starts, starts.shape[0], _I32, "starts"), starts.shape[0] - 1


def tbp_packed_attention_fwd(qkv, starts, n_heads, n_kv_heads, head_dim, out=None, lse=None):
    """qkv [rows, (n_heads + 2 n_kv_heads) head_dim] (q | k | v, rotated), sequence b in rows starts[b] .. starts[b + 1] - 1 -> (out [rows, n_heads*head_dim],
    lse2 [heads, rows]); rows behind the last sequence: zeros and -infinity."""
    rows, dt, ld_out = qkv.shape[0], qkv.dtype, n_heads * head_dim
    at, n = _starts(starts)
    ld_qkv = _matrix(qkv, dt, "qkv", rows, (n_heads + 2 * n_kv_heads) * head_dim)
    given = out, lse
    if out is None:
        out = qkv.new_empty((rows, ld_out))
    else:
        ld_out = _matrix(out, dt, "out", rows, ld_out)
    if lse is None:
        lse = qkv.new_empty((n_heads, rows), dtype=_F32)
    else:
        _vector(lse, n_heads * rows, _F32, "lse")
    _check(lib().tbp_packed_attention_fwd(_dt(qkv), n, rows, n_heads, n_kv_heads, head_dim, at, qkv.data_ptr(), ld_qkv, out.data_ptr(), ld_out, lse.data_ptr(),
                                          _stream_of(qkv.get_device(), starts, *given)))
    return out, lse


def tbp_packed_attention_p1(qkv, out, d_out, lse, starts, n_heads, n_kv_heads, head_dim, dqkv=None, scratch=None):
    """-> dqkv [rows, (n_heads + 2 n_kv_heads) head_dim] (dq | dk | dv, not rotated back)."""
    rows, dt, ld_dqkv = qkv.shape[0], qkv.dtype, (n_heads + 2 * n_kv_heads) * head_dim
    at_starts, n = _starts(starts)
    ld_qkv, ld_out = _matrix(qkv, dt, "qkv", rows, ld_dqkv), _matrix(out, dt, "out", rows, n_heads * head_dim)
    if d_out.shape != out.shape or _matrix(d_out, dt, "d_out", rows, n_heads * head_dim) != ld_out:
        raise TypeError("d_out must have out's shape and leading dimension")
    given = dqkv, scratch
    if dqkv is None:
        dqkv = qkv.new_empty((rows, ld_dqkv))
    else:
        ld_dqkv = _matrix(dqkv, dt, "dqkv", rows, ld_dqkv)
    L = lib()
    need = L.tbp_packed_attention_p1_scratch_bytes(n, rows, n_heads, n_kv_heads, head_dim)
    if scratch is None:
        scratch = qkv.new_empty(need, dtype=torch.uint8)
    at, nbytes = _memory(scratch, "scratch")
    if nbytes < need:
        raise ValueError(f"scratch must have {need} bytes, not {nbytes}")
    _check(L.tbp_packed_attention_p1(_dt(qkv), n, rows, n_heads, n_kv_heads, head_dim, at_starts, qkv.data_ptr(), ld_qkv, out.data_ptr(), d_out.data_ptr(), ld_out,
                                     _vector(lse, n_heads * rows, _F32, "lse"), dqkv.data_ptr(), ld_dqkv, at,
                                     _stream_of(qkv.get_device(), starts, out, d_out, lse, *given)))
    return dqkv


def tbp_packed_attention_plan(n_seqs, rows, n_heads, n_kv_heads, head_dim):
    """How forward and backward-p1 run: a tbp_packed_plan."""
    plan = tbp_packed_plan()
    _check(lib().tbp_packed_attention_plan(n_seqs, rows, n_heads, n_kv_heads, head_dim, C.byref(plan)))
    return plan


# ---- a stash in 8 bits -----------------------------------------------------------------------------------------------------------
class Stash8:
    """`slots` micro-batches [tokens, cols] of one tensor, held in 8 bits with a power of two as scale for every 1024 tokens of a column: a linear layer's inputs or
    output derivatives between backward-p1 and backward-p2 (tbp_stash8_dw), or what a functional operation needs again (get).  A slot that nothing
    was put into holds zeros (the memory is zeroed on the stream that is current now).  dtype: of the tensors that get returns."""

    def __init__(self, tokens, cols, slots=1, dtype=torch.bfloat16, device="cuda"):
        nbytes = lib().tbp_stash8_bytes(slots, tokens, cols)
        if nbytes == 0:
            raise ValueError(f"no stash of {slots} slots of {tokens} tokens of {cols} columns: " + lib().tbp_last_error().decode())
        self.tokens, self.cols, self.slots, self.dtype = tokens, cols, slots, dtype
        self.memory = torch.zeros(nbytes, dtype=torch.uint8, device=device)

    def put(self, slot, x):
        """x [tokens, cols], in the storage type or fp32, into a slot."""
        if x.shape != (self.tokens, self.cols):
            raise TypeError(f"x must be [{self.tokens}, {self.cols}], not {list(x.shape)}")
        _check(lib().tbp_stash8_put(_dt(x), self.slots, self.tokens, self.cols, slot, x.data_ptr(), _matrix(x, x.dtype, "x", self.tokens, self.cols),
                                    self.memory.data_ptr(), _stream_of(x.get_device(), self.memory)))

    def get(self, slot, out=None):
        """-> what the slot holds, [tokens, cols] (out: the tensor to write to)."""
        ld = self.cols
        given = out
        if out is None:
            out = self.memory.new_empty((self.tokens, self.cols), dtype=self.dtype)
        else:
            ld = _matrix(out, out.dtype, "out", self.tokens, self.cols)
        _check(lib().tbp_stash8_get(_dt(out), self.slots, self.tokens, self.cols, slot, self.memory.data_ptr(), out.data_ptr(), ld,
                                    _stream_of(self.memory.get_device(), given)))
        return out


def tbp_stash8_dw(x, dy, first=0, n=None, dw=None, accumulate=False, workspace=None):
    """X^T dY over the slots first .. first + n - 1 (None: to the last one) of two stashes of the same slots and tokens -> dw [x.cols, dy.cols] fp32
    (accumulate: added to the given dw)."""
    if (x.slots, x.tokens) != (dy.slots, dy.tokens):
        raise ValueError(f"stashes of {x.slots} slots of {x.tokens} tokens and of {dy.slots} of {dy.tokens}")
    n = x.slots - first if n is None else n
    ld = dy.cols
    given = dw, workspace
    if dw is None:
        if accumulate:
            raise ValueError("accumulate needs a dw to add to")
        dw = x.memory.new_empty((x.cols, dy.cols), dtype=_F32)
    else:
        ld = _matrix(dw, _F32, "dw", x.cols, dy.cols)
    L = lib()
    need = L.tbp_stash8_dw_workspace_bytes(x.tokens, x.cols, dy.cols, n)
    if workspace is None and need:
        workspace = x.memory.new_empty(need)
    at, nbytes = _memory(workspace, "workspace")
    _check(L.tbp_stash8_dw(x.slots, x.tokens, x.cols, dy.cols, first, n, x.memory.data_ptr(), dy.memory.data_ptr(), dw.data_ptr(), ld, 1 if accumulate else 0,
                           at, nbytes, _stream_of(x.memory.get_device(), dy.memory, *given)))
    return dw


def tbp_stash8_dw_plan(tokens, m, n_out, n):
    """(rows and columns of a workgroup's output tile, shares of the contraction) of tbp_stash8_dw over n slots."""
    out = [C.c_int() for _ in range(2)]
    _check(lib().tbp_stash8_dw_plan(tokens, m, n_out, n, *(C.byref(o) for o in out)))
    return tuple(o.value for o in out)
