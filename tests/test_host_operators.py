"""CPU-only checks of the operators' entry points: every refusal comes from the host, before anything is launched, with a status and a
text; and the sizes that they ask callers for."""
import ctypes as C

import pytest
import torch

import paper_2405_18047_amd as tbp

P = C.c_void_p(1 << 20)                          # an address that nobody may touch, aligned to everything
ODD = C.c_void_p((1 << 20) + 1)
BF16, F32 = tbp.TBP_BF16, tbp.TBP_F32


def _refused(status, word=""):
    text = tbp.lib().tbp_last_error().decode()
    assert status == 1 and text and word in text, (status, text)


WINDOW = dict(dtype=BF16, batch=2, n_heads=4, n_kv_heads=2, seq=100, head_dim=64, window=10, sinks=1, lengths=P, qkv=P, ld_qkv=512, out=P,
              ld_out=256, lse=P, stream=None)
WINDOW_P1 = dict(dtype=BF16, batch=2, n_heads=4, n_kv_heads=2, seq=100, head_dim=64, window=10, sinks=1, lengths=P, qkv=P, ld_qkv=512, out=P,
                 d_out=P, ld_out=256, lse=P, dqkv=P, ld_dqkv=512, scratch=P, stream=None)
DECODE = dict(dtype=BF16, batch=2, n_heads=4, n_kv_heads=2, head_dim=64, window=10, sinks=1, capacity=11, lengths=P, q=P, ld_q=256, cache_k=P,
              cache_v=P, ld_cache=128, out=P, ld_out=256, lse=P, workspace=P, workspace_bytes=1 << 30, stream=None)
ROTARY = dict(dtype=BF16, rows=4, n_heads=2, head_dim=64, rot_dim=32, layout=0, table=P, n_pos=10, positions=None, seq=4, backward=0, x=P,
              ld_x=128, y=C.c_void_p(1 << 21), ld_y=128, stream=None)
APPEND = dict(dtype=BF16, batch=2, n_new=1, n_heads=4, n_kv_heads=2, head_dim=64, rot_dim=32, layout=0, table=P, n_pos=10, lengths=P, qkv=P,
              ld_qkv=512, q_out=P, ld_q=256, cache_k=P, cache_v=P, ld_cache=128, capacity=8, sinks=2, stream=None)
LOGPROBS = dict(dtype=BF16, rows=3, vocab=50, logits=P, ld_logits=50, targets=P, logp=P, entropy=P, lse=P, top=3, top_logp=P, top_ids=P,
                stream=None)
LOGPROBS_P1 = dict(dtype=BF16, rows=3, vocab=50, logits=P, ld_logits=50, targets=P, lse=P, entropy=P, d_logp=P, d_entropy=None, d_logits=P,
                   ld_d=50, stream=None)
LOGPROBS_STEP = dict(dtype=BF16, rows=3, vocab=50, logits=P, ld_logits=50, targets=P, d_logp=P, d_entropy=None, logp=P, entropy=P, lse=P,
                     d_logits=P, ld_d=50, stream=None)

CASES = [("tbp_window_attention_fwd", WINDOW, change) for change in (
    {"dtype": F32}, {"dtype": 9}, {"head_dim": 96}, {"n_kv_heads": 3}, {"n_kv_heads": 0}, {"n_heads": 0}, {"batch": -1}, {"seq": -1},
    {"batch": 1 << 21}, {"seq": (1 << 20) + 1}, {"window": 0}, {"sinks": -1}, {"qkv": None}, {"out": None}, {"lse": None}, {"ld_qkv": 504}, {"ld_qkv": 516},
    {"ld_out": 248}, {"ld_out": 1 << 22}, {"qkv": ODD}, {"out": ODD})]
CASES += [("tbp_window_attention_p1", WINDOW_P1, change) for change in (
    {"dtype": F32}, {"head_dim": 32}, {"window": 0}, {"d_out": None}, {"dqkv": None}, {"scratch": None}, {"scratch": C.c_void_p((1 << 20) + 16)},
    {"ld_dqkv": 256}, {"d_out": ODD}, {"lse": None})]
CASES += [("tbp_window_decode", DECODE, change) for change in (
    {"dtype": F32}, {"head_dim": 80}, {"capacity": 1}, {"capacity": 0}, {"capacity": (1 << 30) + 1}, {"lengths": None}, {"q": None}, {"cache_v": None},
    {"ld_q": 128}, {"ld_cache": 64}, {"ld_cache": 132}, {"q": ODD}, {"window": 0}, {"lse": None},
    {"window": 100000, "workspace": None}, {"window": 100000, "workspace_bytes": 8}, {"window": 100000, "workspace": C.c_void_p((1 << 20) + 16)})]
CASES += [("tbp_rotary", ROTARY, change) for change in (
    {"dtype": 5}, {"rows": -1}, {"rot_dim": 0}, {"rot_dim": 31}, {"rot_dim": 66}, {"layout": 2}, {"table": None}, {"table": ODD}, {"n_pos": 0},
    {"seq": 0}, {"ld_x": 127}, {"ld_y": 64}, {"x": None}, {"y": None}, {"x": ODD}, {"y": P, "ld_y": 130})]
CASES += [("tbp_rotary_append", APPEND, change) for change in (
    {"dtype": 5}, {"batch": -1}, {"n_new": -1}, {"batch": 1 << 20, "n_new": 1 << 20}, {"n_kv_heads": 3}, {"capacity": 2}, {"sinks": -1}, {"ld_qkv": 511},
    {"ld_q": 255}, {"ld_cache": 127}, {"lengths": None}, {"cache_k": None}, {"q_out": None}, {"cache_v": ODD}, {"rot_dim": 3})]
CASES += [("tbp_logprobs", LOGPROBS, change) for change in (
    {"dtype": 2}, {"rows": -1}, {"vocab": 0}, {"vocab": (1 << 24) + 1}, {"ld_logits": 49}, {"logits": None}, {"logits": ODD}, {"targets": None},
    {"logp": None}, {"entropy": None}, {"lse": None}, {"top": -1}, {"top": 65}, {"top": 51}, {"top_ids": None}, {"top_logp": None})]
CASES += [("tbp_logprobs_p1", LOGPROBS_P1, change) for change in (
    {"dtype": 2}, {"ld_d": 49}, {"d_logp": None}, {"lse": None}, {"entropy": None}, {"d_logits": None}, {"d_logits": ODD}, {"ld_d": 51}, {"targets": None})]
CASES += [("tbp_logprobs_step", LOGPROBS_STEP, change) for change in (
    {"dtype": 2}, {"ld_d": 49}, {"d_logp": None}, {"logp": None}, {"d_logits": None}, {"ld_logits": 51}, {"targets": None})]


@pytest.mark.parametrize("name,good,change", CASES, ids=lambda v: v if isinstance(v, str) else ",".join(v) if len(v) < 4 else "")
def test_bad_arguments_are_refused(name, good, change):
    _refused(getattr(tbp.lib(), name)(*{**good, **change}.values()))


@pytest.mark.parametrize("name,good,change", [
    ("tbp_window_attention_fwd", WINDOW, {"batch": 0}), ("tbp_window_attention_fwd", WINDOW, {"seq": 0}), ("tbp_window_attention_p1", WINDOW_P1, {"seq": 0}),
    ("tbp_window_decode", DECODE, {"batch": 0}), ("tbp_rotary", ROTARY, {"rows": 0}), ("tbp_rotary", ROTARY, {"n_heads": 0}),
    ("tbp_rotary_append", APPEND, {"n_new": 0}), ("tbp_logprobs", LOGPROBS, {"rows": 0}), ("tbp_logprobs_p1", LOGPROBS_P1, {"rows": 0}),
    ("tbp_logprobs_step", LOGPROBS_STEP, {"rows": 0})])
def test_empty_calls_do_nothing(name, good, change):
    assert getattr(tbp.lib(), name)(*{**good, **change}.values()) == 0


@pytest.mark.parametrize("change", [{"n_pos": 0}, {"rot_dim": 3}, {"rot_dim": 5000}, {"base": 0.0}, {"base": float("nan")}, {"table": None},
                                    {"scale": (4, 1, 1, 2, 1, 1)}, {"scale": (1, 0, 1, 2, 1, 1)}, {"scale": (2, 2, 1, 2, 1, 1), "rot_dim": 2},
                                    {"scale": (3, 2, 2, 2, 1, 1)}, {"scale": (3, 2, 1, 2, 0, 1)}, {"scale": (0, 1, 1, 2, 1, -1)},
                                    {"scale": (1, float("nan"), 1, 2, 1, 1)}], ids=str)
def test_bad_rotary_tables_are_refused(change):
    a = {"n_pos": 4, "rot_dim": 8, "base": 1e4, "scale": None, "table": P, **change}
    sc = C.byref(tbp.tbp_rotary_scale(*a["scale"])) if a["scale"] else None
    _refused(tbp.lib().tbp_rotary_table(a["n_pos"], a["rot_dim"], a["base"], sc, a["table"], None))


def test_bad_gradient_lists_are_refused():
    L = tbp.lib()
    src, cnt = (C.c_void_p * 2)(1 << 20, 1 << 21), (C.c_int64 * 2)(10, 10)
    null, odd, neg = (C.c_void_p * 2)(1 << 20, None), (C.c_void_p * 2)(1 << 20, (1 << 21) + 1), (C.c_int64 * 2)(10, -1)
    for args in ((7, 2, src, cnt, P, P), (F32, -1, src, cnt, P, P), (F32, 2, None, cnt, P, P), (F32, 2, src, None, P, P), (F32, 2, null, cnt, P, P),
                 (F32, 2, odd, cnt, P, P), (F32, 2, src, neg, P, P), (F32, 2, src, cnt, None, P), (F32, 2, src, cnt, P, None), (F32, 2, src, cnt, P, ODD)):
        _refused(L.tbp_grad_sumsq(*args, None))
    for args in ((F32, 7, 2, src, src, cnt, None, 1.0, P, P), (F32, F32, 2, src, None, cnt, None, 1.0, P, P), (F32, F32, 2, src, null, cnt, None, 1.0, P, P),
                 (F32, F32, 2, src, odd, cnt, None, 1.0, P, P), (F32, BF16, 2, src, src, cnt, None, 1.0, P, P), (F32, F32, 2, src, src, cnt, ODD, 1.0, P, P),
                 (F32, F32, 2, src, src, cnt, None, -1.0, P, P), (F32, F32, 2, src, src, cnt, None, float("nan"), P, P), (F32, F32, 2, src, src, cnt, None, 1.0, P, None)):
        _refused(L.tbp_grad_clip(*args, None))


def test_sizes_that_callers_are_asked_for():
    L = tbp.lib()
    # the row sums at least, and room for a bounded number of parts of key blocks; nothing of the size of the scores
    for b, h, kv, s, dh, w, k in ((1, 32, 8, 8192, 128, 2048, 4), (4, 12, 4, 1001, 64, 300, 3), (1, 1, 1, 1, 64, 1, 0), (2, 8, 1, 100000, 128, 512, 1000),
                              (1, 64, 8, 1 << 20, 128, 1, 1 << 20), (1, 1, 1, 1 << 20, 64, 4096, 1 << 19)):
        got = L.tbp_window_attention_p1_scratch_bytes(b, h, kv, s, dh, w, k)
        assert b * h * s * 4 <= got < b * h * s * 4 + (1 << 30)
    assert L.tbp_window_attention_p1_scratch_bytes(0, 32, 8, 8192, 128, 2048, 4) == 0 == L.tbp_window_attention_p1_scratch_bytes(1, 3, 2, 8, 128, 1, 4)
    assert L.tbp_window_decode_workspace_bytes(64, 32, 8, 128, 4096, 4) < 1 << 28
    assert L.tbp_rotary_table_bytes(10, 8) == 320 and L.tbp_rotary_table_bytes(0, 8) == 0
    assert L.tbp_grad_workspace_bytes(0) > 0 and L.tbp_grad_workspace_bytes(1000) >= L.tbp_grad_workspace_bytes(1)


def test_the_binding_refuses_other_types_and_shapes():
    x, t = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros((4, 2, 2))
    with pytest.raises(TypeError):
        tbp.tbp_logprobs(x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(TypeError):
        tbp.tbp_rotary(x, 1, 8, t.double())
    with pytest.raises(TypeError):
        tbp.tbp_rotary(x.t(), 1, 4, t, seq=4)
    with pytest.raises(ValueError):
        tbp.tbp_window_attention_fwd(x, 3, 1, 1, 64, 2)
    with pytest.raises(TypeError):
        tbp.GradList([x, x.float()])
    with pytest.raises(ValueError):
        tbp.GradList([x], [x[:2]])
    with pytest.raises(TypeError):
        tbp.tbp_window_decode(x, x, x, torch.zeros(4, dtype=torch.int32), 1, 1, 64, 2)


def test_a_gradient_list_refuses_tensors_that_moved():
    g, o = torch.zeros(8), torch.zeros(8)
    moved = tbp.GradList([g], [o])
    o.data = torch.zeros(8)
    for call in (moved.sumsq, lambda: moved.clip(1.0)):
        with pytest.raises(RuntimeError, match="other memory"):
            call()


def _bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _good_calls():
    """One call of every operator that takes tensors of the caller's, with arguments that fit: 6 tokens, 4 query heads on 2 key heads of 64."""
    table = torch.zeros((16, 32, 2))
    return {
        "window_fwd": (tbp.tbp_window_attention_fwd, dict(qkv=_bf(6, 512), seq=3, n_heads=4, n_kv_heads=2, head_dim=64, window=2, lengths=_i32(2), out=_bf(6, 256),
                                                          lse=torch.zeros((2, 4, 3)))),
        "window_p1": (tbp.tbp_window_attention_p1, dict(qkv=_bf(6, 512), out=_bf(6, 256), d_out=_bf(6, 256), lse=torch.zeros((2, 4, 3)), seq=3, n_heads=4,
                                                        n_kv_heads=2, head_dim=64, window=2, lengths=_i32(2), dqkv=_bf(6, 512),
                                                        scratch=torch.zeros(1 << 20, dtype=torch.uint8))),
        "decode": (tbp.tbp_window_decode, dict(q=_bf(2, 256), cache_k=_bf(2, 8, 128), cache_v=_bf(2, 8, 128), lengths=_i32(2), n_heads=4, n_kv_heads=2, head_dim=64,
                                               window=9000, out=_bf(2, 256), lse=torch.zeros((2, 4)), workspace=torch.zeros(1 << 22, dtype=torch.uint8))),
        "rotary": (tbp.tbp_rotary, dict(x=_bf(6, 384), n_heads=6, head_dim=64, table=table, positions=_i32(6), out=_bf(6, 384))),
        "append": (tbp.tbp_rotary_append, dict(qkv=_bf(6, 512), n_heads=4, n_kv_heads=2, head_dim=64, table=table, lengths=_i32(2), cache_k=_bf(2, 8, 128),
                                               cache_v=_bf(2, 8, 128), q_out=_bf(6, 256))),
        "logprobs": (tbp.tbp_logprobs, dict(logits=_bf(6, 50), targets=_i32(6))),
        "logprobs_p1": (tbp.tbp_logprobs_p1, dict(logits=_bf(6, 50), targets=_i32(6), lse=torch.zeros(6), entropy=torch.zeros(6), d_logp=torch.zeros(6),
                                                  d_entropy=torch.zeros(6), out=_bf(6, 50))),
        "logprobs_step": (tbp.tbp_logprobs_step, dict(logits=_bf(6, 50), targets=_i32(6), d_logp=torch.zeros(6), d_entropy=torch.zeros(6), out=_bf(6, 50))),
    }


def _beside(rows, columns, ld):
    """A view of `columns` columns of an array of `ld`: its leading dimension would cover more."""
    return _bf(rows, ld)[:, :columns]


@pytest.mark.parametrize("name,what,given", [
    ("window_fwd", "qkv", _beside(6, 504, 1024)), ("window_fwd", "out", _bf(5, 256)), ("window_fwd", "out", _beside(6, 248, 512)),
    ("window_p1", "qkv", _beside(6, 448, 512)), ("window_p1", "out", _bf(5, 256)), ("window_p1", "out", _beside(6, 128, 256)), ("window_p1", "d_out", _bf(5, 256)),
    ("window_p1", "dqkv", _bf(5, 512)), ("window_p1", "dqkv", _beside(6, 384, 512)), ("decode", "q", _beside(2, 128, 256)), ("decode", "out", _bf(1, 256)),
    ("decode", "out", _beside(2, 64, 256)), ("rotary", "x", _beside(6, 256, 512)), ("rotary", "out", _bf(5, 384)), ("rotary", "out", _beside(6, 256, 384)),
    ("append", "qkv", _beside(6, 384, 512)), ("append", "q_out", _bf(2, 256)), ("append", "q_out", _beside(6, 192, 256)), ("logprobs_p1", "out", _bf(5, 50)),
    ("logprobs_p1", "out", _beside(6, 49, 64)), ("logprobs_step", "out", _bf(5, 50)), ("logprobs_step", "out", _beside(6, 49, 64))],
    ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v.shape)))
def test_matrices_that_a_call_would_pass_the_end_of_are_refused(name, what, given):
    call, good = _good_calls()[name]
    if (name, what) == ("window_p1", "out"):
        good["d_out"] = given
    with pytest.raises(TypeError, match=what):
        call(**{**good, what: given})


def test_scratch_and_workspace_that_are_too_small_are_refused():
    """The backward's scratch (whose size the C entry point is not told) and the decode's workspace, also where a tensor stands for more entries than it has memory."""
    call, good = _good_calls()["window_p1"]
    need = tbp.lib().tbp_window_attention_p1_scratch_bytes(2, 4, 2, 3, 64, 2, 0)
    assert need > 1
    for scratch in (torch.zeros(need - 1, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8).expand(need), torch.zeros(need // 4, dtype=torch.uint8)):
        with pytest.raises((TypeError, ValueError), match="scratch"):
            call(**{**good, "scratch": scratch})
    call, good = _good_calls()["decode"]
    need = tbp.lib().tbp_window_decode_workspace_bytes(2, 4, 2, 64, 9000, 0)
    assert need > 1
    with pytest.raises(TypeError, match="workspace"):
        call(**{**good, "workspace": torch.zeros(1, dtype=torch.uint8).expand(need)})


@pytest.mark.parametrize("name", list(_good_calls()))
def test_tensors_of_the_host_are_refused(name):
    """Their addresses mean nothing to a kernel."""
    call, good = _good_calls()[name]
    with pytest.raises(TypeError, match="GPU"):
        call(**good)


def test_gradients_of_the_host_are_refused():
    some = tbp.GradList([torch.zeros(8)])
    for call in (some.sumsq, lambda: some.clip(1.0)):
        with pytest.raises(TypeError, match="GPU"):
            call()


def test_rotary_rows_of_no_position_are_refused():
    """Neither positions nor a length of the sequences: one sequence, which the table has to cover; it does not start again behind the table's end."""
    table = torch.zeros((5, 32, 2))
    with pytest.raises(ValueError, match="seq"):
        tbp.tbp_rotary(_bf(6, 384), 6, 64, table)
    with pytest.raises(ValueError, match="seq"):
        tbp.tbp_rotary(_bf(6, 384), 6, 64, table, seq=0)
    with pytest.raises(TypeError, match="GPU"):                  # (as many rows as positions: nothing but the place of the tensors is wrong)
        tbp.tbp_rotary(_bf(5, 384), 6, 64, table)


def test_new_memory_is_the_current_device_s(monkeypatch):
    """A process that has chosen its GPU gets workspaces and tables there: a device without an index is torch's current one."""
    asked = []

    def note(*shape, **kw):
        asked.append(torch.device(kw["device"]))
        raise InterruptedError

    monkeypatch.setattr(torch, "zeros", note)
    monkeypatch.setattr(torch, "empty", note)
    for call in (lambda: tbp.tbp_window_decode_workspace(2, 4, 2, 64, 9000), lambda: tbp.tbp_rotary_table(8, 64, 1e4), lambda: tbp.GradList([])):
        with pytest.raises(InterruptedError):
            call()
    assert asked == [torch.device("cuda")] * 3


@pytest.mark.parametrize("n_pos,rot_dim", [(1 << 26, 128), ((1 << 31) - 1, 4), ((1 << 31) - 1, 4096)])
def test_rotary_tables_of_more_entries_than_a_launch_has_threads_are_refused(n_pos, rot_dim):
    _refused(tbp.lib().tbp_rotary_table(n_pos, rot_dim, 1e4, None, P, None), "entries")
