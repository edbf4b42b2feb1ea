"""Binding of the operators for long contexts, the last stage and serving: sliding-window attention with sinks, rotary
positions, log probabilities of tokens, the norm of all gradients with clipping.

As in binding.py: argument marshalling only, on torch's current stream; outputs and workspaces are allocated where the caller
passes none.  Index tensors (lengths, positions, targets) are int32 on the device.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import _check, _dt, _ptr, _stream, lib

__all__ = [
    "TBP_ROTARY_HALF", "TBP_ROTARY_INTERLEAVED", "TBP_ROTARY_PLAIN", "TBP_ROTARY_LINEAR", "TBP_ROTARY_BASE", "TBP_ROTARY_RAMP",
    "tbp_rotary_scale", "tbp_rotary_table", "tbp_rotary", "tbp_rotary_append", "tbp_window_attention_fwd", "tbp_window_attention_p1",
    "tbp_window_decode_workspace", "tbp_window_decode", "tbp_logprobs", "tbp_logprobs_p1", "tbp_logprobs_step", "GradList",
]

TBP_ROTARY_HALF, TBP_ROTARY_INTERLEAVED = 0, 1
TBP_ROTARY_PLAIN, TBP_ROTARY_LINEAR, TBP_ROTARY_BASE, TBP_ROTARY_RAMP = 0, 1, 2, 3


class tbp_rotary_scale(C.Structure):
    _fields_ = [("scaling", C.c_int32), ("factor", C.c_float), ("low", C.c_float), ("high", C.c_float), ("original", C.c_float),
                ("magnitude", C.c_float)]


def _index(t, n, what):
    """An int32 vector of n entries, or None."""
    if t is None:
        return None
    if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise TypeError(f"{what} must be a contiguous int32 tensor of {n} entries")
    return _ptr(t)


def _floats(t, n, what):
    if t is None:
        return None
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{what} must be a contiguous float32 tensor of {n} entries")
    return _ptr(t)


def _matrix(t, what):
    """The leading dimension of a tensor whose rows are contiguous."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise TypeError(f"{what} must be a matrix with contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _like(t, ref, what):
    if t.dtype != ref.dtype or t.device != ref.device:
        raise TypeError(f"{what} must have type {ref.dtype} on {ref.device}")
    return t


def _workspace(nbytes, device):
    """A uint8 tensor (256-byte aligned, as torch's allocations on the device are), or None for nothing."""
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


# ---- sliding-window attention ------------------------------------------------------------------------------------------
def _sequences(rows, seq):
    if seq < 1 or rows % seq:
        raise ValueError(f"{rows} rows are no whole sequences of {seq}")
    return rows // seq


def tbp_window_attention_fwd(qkv, seq, n_heads, n_kv_heads, head_dim, window, sinks=0, lengths=None, out=None, lse=None):
    """qkv [batch*seq, (n_heads + 2 n_kv_heads) head_dim] (q | k | v, rotated) -> (out [batch*seq, n_heads*head_dim], lse2 [batch, heads, seq])."""
    batch = _sequences(qkv.shape[0], seq)
    out = torch.empty((qkv.shape[0], n_heads * head_dim), dtype=qkv.dtype, device=qkv.device) if out is None else _like(out, qkv, "out")
    lse = torch.empty((batch, n_heads, seq), dtype=torch.float32, device=qkv.device) if lse is None else lse
    _check(lib().tbp_window_attention_fwd(_dt(qkv), batch, n_heads, n_kv_heads, seq, head_dim, window, sinks, _index(lengths, batch, "lengths"),
                                          _ptr(qkv), _matrix(qkv, "qkv"), _ptr(out), _matrix(out, "out"), _floats(lse, batch * n_heads * seq, "lse"),
                                          _stream()))
    return out, lse


def tbp_window_attention_p1(qkv, out, d_out, lse, seq, n_heads, n_kv_heads, head_dim, window, sinks=0, lengths=None, dqkv=None, scratch=None):
    """-> dqkv [batch*seq, (n_heads + 2 n_kv_heads) head_dim] (dq | dk | dv, not rotated back)."""
    batch = _sequences(qkv.shape[0], seq)
    _like(out, qkv, "out"), _like(d_out, qkv, "d_out")
    if _matrix(d_out, "d_out") != _matrix(out, "out") or d_out.shape != out.shape:
        raise TypeError("d_out must have out's shape and leading dimension")
    dqkv = torch.empty((qkv.shape[0], (n_heads + 2 * n_kv_heads) * head_dim), dtype=qkv.dtype, device=qkv.device) if dqkv is None else _like(dqkv, qkv, "dqkv")
    if scratch is None:
        scratch = _workspace(lib().tbp_window_attention_p1_scratch_bytes(batch, n_heads, n_kv_heads, seq, head_dim, window, sinks), qkv.device)
    _check(lib().tbp_window_attention_p1(_dt(qkv), batch, n_heads, n_kv_heads, seq, head_dim, window, sinks, _index(lengths, batch, "lengths"),
                                         _ptr(qkv), _matrix(qkv, "qkv"), _ptr(out), _ptr(d_out), _matrix(out, "out"),
                                         _floats(lse, batch * n_heads * seq, "lse"), _ptr(dqkv), _matrix(dqkv, "dqkv"), _ptr(scratch), _stream()))
    return dqkv


def tbp_window_decode_workspace(batch, n_heads, n_kv_heads, head_dim, window, sinks=0, device="cuda:0"):
    """The workspace of tbp_window_decode calls of these sizes (which must not overlap), or None where they need none."""
    return _workspace(lib().tbp_window_decode_workspace_bytes(batch, n_heads, n_kv_heads, head_dim, window, sinks), device)


def _cache(t, batch, width, what):
    if t.dim() != 3 or t.shape[0] != batch or t.shape[2] != width or t.stride(2) != 1 or t.stride(0) != t.shape[1] * t.stride(1):
        raise TypeError(f"{what} must be [batch, capacity, n_kv_heads*head_dim] with contiguous rows of one distance")
    return t


def tbp_window_decode(q, cache_k, cache_v, lengths, n_heads, n_kv_heads, head_dim, window, sinks=0, out=None, lse=None, workspace=None):
    """q [batch, n_heads*head_dim] of the token at position lengths[b] - 1 over caches [batch, capacity, n_kv_heads*head_dim] ->
    (out [batch, n_heads*head_dim], lse2 [batch, heads])."""
    batch, width = q.shape[0], n_kv_heads * head_dim
    _cache(_like(cache_k, q, "cache_k"), batch, width, "cache_k"), _cache(_like(cache_v, q, "cache_v"), batch, width, "cache_v")
    if cache_k.shape != cache_v.shape or cache_k.stride() != cache_v.stride():
        raise TypeError("cache_k and cache_v must have one shape and stride")
    out = torch.empty((batch, n_heads * head_dim), dtype=q.dtype, device=q.device) if out is None else _like(out, q, "out")
    lse = torch.empty((batch, n_heads), dtype=torch.float32, device=q.device) if lse is None else lse
    if workspace is None:
        workspace = tbp_window_decode_workspace(batch, n_heads, n_kv_heads, head_dim, window, sinks, q.device)
    _check(lib().tbp_window_decode(_dt(q), batch, n_heads, n_kv_heads, head_dim, window, sinks, cache_k.shape[1], _index(lengths, batch, "lengths"),
                                   _ptr(q), _matrix(q, "q"), _ptr(cache_k), _ptr(cache_v), cache_k.stride(1), _ptr(out), _matrix(out, "out"),
                                   _floats(lse, batch * n_heads, "lse"), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream()))
    return out, lse


# ---- rotary positions ----------------------------------------------------------------------------------------------------
def tbp_rotary_table(n_pos, rot_dim, base, scaling=TBP_ROTARY_PLAIN, factor=1.0, low=1.0, high=32.0, original=4096.0, magnitude=1.0,
                     device="cuda:0"):
    """-> table [n_pos, rot_dim/2, 2] of cosines and sines."""
    t = torch.empty((n_pos, rot_dim // 2, 2), dtype=torch.float32, device=device)
    sc = tbp_rotary_scale(scaling, factor, low, high, original, magnitude)
    _check(lib().tbp_rotary_table(n_pos, rot_dim, base, C.byref(sc), _ptr(t), _stream()))
    return t


def _table(table):
    if table.dtype != torch.float32 or table.dim() != 3 or table.shape[2] != 2 or not table.is_contiguous():
        raise TypeError("the table must be a contiguous float32 tensor [n_pos, rot_dim/2, 2]")
    return table.shape[0], 2 * table.shape[1]


def tbp_rotary(x, n_heads, head_dim, table, positions=None, seq=None, layout=TBP_ROTARY_HALF, backward=False, out=None):
    """The first n_heads*head_dim columns of x [rows, ld], turned (backward: the derivative).  seq: tokens per sequence, where no positions
    are given.  out: new [rows, n_heads*head_dim], or the tensor to write to (x itself: in place)."""
    n_pos, rot_dim = _table(table)
    rows = x.shape[0]
    out = torch.empty((rows, n_heads * head_dim), dtype=x.dtype, device=x.device) if out is None else _like(out, x, "out")
    _check(lib().tbp_rotary(_dt(x), rows, n_heads, head_dim, rot_dim, layout, _ptr(table), n_pos, _index(positions, rows, "positions"),
                            (seq or n_pos) if positions is None else 1, 1 if backward else 0, _ptr(x), _matrix(x, "x"), _ptr(out),
                            _matrix(out, "out"), _stream()))
    return out


def tbp_rotary_append(qkv, n_heads, n_kv_heads, head_dim, table, lengths, cache_k, cache_v, sinks=0, layout=TBP_ROTARY_HALF, q_out=None):
    """New tokens qkv [batch*n_new, (n_heads + 2 n_kv_heads) head_dim], the last ones of sequences of `lengths`: k (rotated) and v into the
    caches [batch, capacity, n_kv_heads*head_dim]; -> q rotated [batch*n_new, n_heads*head_dim]."""
    n_pos, rot_dim = _table(table)
    batch, width = lengths.shape[0], n_kv_heads * head_dim
    n_new = 0 if batch == 0 else qkv.shape[0] // batch
    if n_new * batch != qkv.shape[0]:
        raise ValueError(f"{qkv.shape[0]} rows are no whole number of tokens for {batch} sequences")
    _cache(_like(cache_k, qkv, "cache_k"), batch, width, "cache_k"), _cache(_like(cache_v, qkv, "cache_v"), batch, width, "cache_v")
    if cache_k.shape != cache_v.shape or cache_k.stride() != cache_v.stride():
        raise TypeError("cache_k and cache_v must have one shape and stride")
    q_out = torch.empty((qkv.shape[0], n_heads * head_dim), dtype=qkv.dtype, device=qkv.device) if q_out is None else _like(q_out, qkv, "q_out")
    _check(lib().tbp_rotary_append(_dt(qkv), batch, n_new, n_heads, n_kv_heads, head_dim, rot_dim, layout, _ptr(table), n_pos,
                                   _index(lengths, batch, "lengths"), _ptr(qkv), _matrix(qkv, "qkv"), _ptr(q_out), _matrix(q_out, "q_out"),
                                   _ptr(cache_k), _ptr(cache_v), cache_k.stride(1), cache_k.shape[1], sinks, _stream()))
    return q_out


# ---- log probabilities -----------------------------------------------------------------------------------------------------
def _rows(n, device):
    return torch.empty(n, dtype=torch.float32, device=device)


def tbp_logprobs(logits, targets, top=0, workspace=None):
    """logits [rows, vocab], targets [rows] (int32; outside the vocabulary: left out) -> (logp, entropy, lse), each [rows] fp32, and with top > 0
    (top_logp [rows, top] fp32, top_ids [rows, top] int32) behind them."""
    rows, vocab = logits.shape
    logp, entropy, lse = (_rows(rows, logits.device) for _ in range(3))
    top_logp = torch.empty((rows, top), dtype=torch.float32, device=logits.device) if top > 0 else None
    top_ids = torch.empty((rows, top), dtype=torch.int32, device=logits.device) if top > 0 else None
    if workspace is None:
        workspace = _workspace(lib().tbp_logprobs_workspace_bytes(rows, vocab, top), logits.device)
    _check(lib().tbp_logprobs(_dt(logits), rows, vocab, _ptr(logits), _matrix(logits, "logits"), _index(targets, rows, "targets"), _ptr(logp),
                              _ptr(entropy), _ptr(lse), top, _ptr(top_logp), _ptr(top_ids), _ptr(workspace),
                              0 if workspace is None else workspace.numel(), _stream()))
    return (logp, entropy, lse, top_logp, top_ids) if top > 0 else (logp, entropy, lse)


def tbp_logprobs_p1(logits, targets, lse, entropy, d_logp, d_entropy=None, out=None):
    """-> the derivative of the logits [rows, vocab] (out: the tensor to write to, logits itself allowed)."""
    rows, vocab = logits.shape
    out = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device) if out is None else _like(out, logits, "out")
    _check(lib().tbp_logprobs_p1(_dt(logits), rows, vocab, _ptr(logits), _matrix(logits, "logits"), _index(targets, rows, "targets"),
                                 _floats(lse, rows, "lse"), _floats(entropy, rows, "entropy"), _floats(d_logp, rows, "d_logp"),
                                 _floats(d_entropy, rows, "d_entropy"), _ptr(out), _matrix(out, "out"), _stream()))
    return out


def tbp_logprobs_step(logits, targets, d_logp, d_entropy=None, out=None, workspace=None):
    """Forward and derivative in one pass -> (logp, entropy, lse, d_logits)."""
    rows, vocab = logits.shape
    logp, entropy, lse = (_rows(rows, logits.device) for _ in range(3))
    out = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device) if out is None else _like(out, logits, "out")
    if workspace is None:
        workspace = _workspace(lib().tbp_logprobs_workspace_bytes(rows, vocab, 0), logits.device)
    _check(lib().tbp_logprobs_step(_dt(logits), rows, vocab, _ptr(logits), _matrix(logits, "logits"), _index(targets, rows, "targets"),
                                   _floats(d_logp, rows, "d_logp"), _floats(d_entropy, rows, "d_entropy"), _ptr(logp), _ptr(entropy), _ptr(lse),
                                   _ptr(out), _matrix(out, "out"), _ptr(workspace), 0 if workspace is None else workspace.numel(), _stream()))
    return logp, entropy, lse, out


# ---- the norm over gradient tensors, and clipping --------------------------------------------------------------------------
class GradList:
    """The gradient tensors of a stage (or of anything else), of one type, and where they go when they are clipped: into themselves, or
    into tensors of the same sizes and of one type.  Keeps the tensors, their addresses and a workspace; calls of one list must not overlap.

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
        self.device = grads[0].device if n else torch.device("cuda:0")
        self._src = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in grads])
        self._dst = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in outs])
        self._counts = (C.c_int64 * max(n, 1))(*[t.numel() for t in grads])
        self._ws = torch.empty(lib().tbp_grad_workspace_bytes(n), dtype=torch.uint8, device=self.device)

    def sumsq(self, out=None):
        """The sum of squares [1] float64 (stages of a pipeline add theirs up before they clip)."""
        out = torch.empty(1, dtype=torch.float64, device=self.device) if out is None else out
        if out.dtype != torch.float64:
            raise TypeError("out must be float64")
        _check(lib().tbp_grad_sumsq(self._dt, self._n, self._src, self._counts, _ptr(out), _ptr(self._ws), _stream()))
        return out

    def clip(self, max_norm, sumsq=None, norm=None):
        """Writes the outputs; -> the norm [1] float32.  sumsq: [1] float64, computed here where none is given."""
        norm = torch.empty(1, dtype=torch.float32, device=self.device) if norm is None else norm
        if sumsq is not None and sumsq.dtype != torch.float64:
            raise TypeError("sumsq must be float64")
        _check(lib().tbp_grad_clip(self._dt, self._odt, self._n, self._src, self._dst, self._counts, _ptr(sumsq), max_norm, _floats(norm, 1, "norm"),
                                   _ptr(self._ws), _stream()))
        return norm
