"""CPU-only checks of the entry points around packed documents: every refusal comes from the host, before anything is launched, with a status and a
text; and the sizes that they ask callers for."""
import ctypes as C

import pytest
import torch

import paper_2405_18047_amd as tbp

P = C.c_void_p(1 << 20)                          # an address that nobody may touch, aligned to everything
P2 = C.c_void_p(1 << 21)
ODD = C.c_void_p((1 << 20) + 1)
BF16, F32 = tbp.TBP_BF16, tbp.TBP_F32
NAN = float("nan")


def _refused(status, word=""):
    text = tbp.lib().tbp_last_error().decode()
    assert status == 1 and text and word in text, (status, text)


NORM = dict(dtype=BF16, rows=4, n_heads=2, n_kv_heads=1, head_dim=64, eps=1e-5, gq=P, gk=P, rot_dim=32, layout=0, table=P, n_pos=10, positions=None, seq=4,
            x=P, ld_x=192, y=P2, ld_y=192, stream=None)
NORM_P1 = dict(dtype=BF16, rows=4, n_heads=2, n_kv_heads=1, head_dim=64, eps=1e-5, gq=P, gk=P, rot_dim=32, layout=0, table=P, n_pos=10, positions=None, seq=4,
               dy=P, ld_dy=192, x=P2, ld_x=192, dx=P, ld_dx=192, partials=P, stream=None)
APPEND = dict(dtype=BF16, batch=2, n_new=1, n_heads=4, n_kv_heads=2, head_dim=64, eps=1e-5, gq=P, gk=P, rot_dim=32, layout=0, table=P, n_pos=10, lengths=P, qkv=P,
              ld_qkv=512, q_out=P, ld_q=256, cache_k=P, cache_v=P, ld_cache=128, capacity=8, sinks=2, stream=None)
PACKED = dict(dtype=BF16, n_seqs=3, rows=100, n_heads=4, n_kv_heads=2, head_dim=64, starts=P, qkv=P, ld_qkv=512, out=P, ld_out=256, lse=P, stream=None)
PACKED_P1 = dict(dtype=BF16, n_seqs=3, rows=100, n_heads=4, n_kv_heads=2, head_dim=64, starts=P, qkv=P, ld_qkv=512, out=P, d_out=P, ld_out=256, lse=P, dqkv=P,
                 ld_dqkv=512, scratch=P, stream=None)
PUT = dict(dtype=BF16, slots=2, tokens=100, cols=50, slot=1, x=P, ld_x=50, stash=P, stream=None)
GET = dict(dtype=BF16, slots=2, tokens=100, cols=50, slot=1, stash=P, y=P, ld_y=50, stream=None)
DW = dict(slots=4, tokens=100, m=50, n_out=60, first=1, n=2, x=P, dy=P, dw=P, ld_dw=60, accumulate=0, workspace=P, workspace_bytes=1 << 40, stream=None)

CASES = [("tbp_qk_norm", NORM, change) for change in (
    {"dtype": 5}, {"rows": -1}, {"n_heads": -1}, {"n_kv_heads": -1}, {"head_dim": 0}, {"head_dim": 63}, {"head_dim": 514, "ld_x": 2000, "ld_y": 2000}, {"eps": -1.0}, {"eps": NAN},
    {"gq": None}, {"gk": None}, {"gq": ODD}, {"gk": ODD}, {"rot_dim": 31}, {"rot_dim": 66}, {"rot_dim": -2}, {"layout": 2}, {"table": None}, {"table": ODD}, {"n_pos": 0},
    {"seq": 0}, {"ld_x": 191}, {"ld_y": 191}, {"x": None}, {"y": None}, {"x": ODD}, {"y": P, "ld_y": 200}, {"n_heads": 1 << 25})]
CASES += [("tbp_qk_norm_p1", NORM_P1, change) for change in (
    {"dtype": 5}, {"rows": -1}, {"head_dim": 63}, {"eps": NAN}, {"gk": None}, {"rot_dim": 3}, {"table": None}, {"seq": 0}, {"ld_dy": 191}, {"ld_x": 191}, {"ld_dx": 191},
    {"dy": None}, {"x": None}, {"dx": None}, {"partials": None}, {"dy": ODD}, {"partials": ODD}, {"ld_dx": 200}, {"dx": P2})]
CASES += [("tbp_qk_norm_append", APPEND, change) for change in (
    {"dtype": 5}, {"batch": -1}, {"n_new": -1}, {"batch": 1 << 20, "n_new": 1 << 20}, {"n_kv_heads": 3}, {"capacity": 2}, {"sinks": -1}, {"ld_qkv": 511},
    {"ld_q": 255}, {"ld_cache": 127}, {"lengths": None}, {"cache_k": None}, {"q_out": None}, {"cache_v": ODD}, {"rot_dim": 3}, {"gq": None}, {"eps": -1.0}, {"head_dim": 600})]
CASES += [("tbp_packed_attention_fwd", PACKED, change) for change in (
    {"dtype": F32}, {"head_dim": 96}, {"n_kv_heads": 3}, {"n_heads": 0}, {"n_seqs": -1}, {"rows": -1}, {"rows": (1 << 22) + 1}, {"n_seqs": (1 << 20) + 1},
    {"n_heads": 1 << 14, "n_kv_heads": 1, "rows": 1 << 22}, {"starts": None}, {"qkv": None}, {"out": None}, {"lse": None}, {"ld_qkv": 504}, {"ld_qkv": 516}, {"ld_out": 248},
    {"ld_out": 1 << 22}, {"qkv": ODD}, {"out": ODD})]
CASES += [("tbp_packed_attention_p1", PACKED_P1, change) for change in (
    {"dtype": F32}, {"head_dim": 32}, {"d_out": None}, {"dqkv": None}, {"scratch": None}, {"scratch": C.c_void_p((1 << 20) + 16)}, {"ld_dqkv": 256}, {"d_out": ODD}, {"lse": None})]
CASES += [("tbp_stash8_put", PUT, change) for change in (
    {"dtype": 2}, {"slots": -1}, {"slots": 1}, {"slot": -1}, {"slot": 2}, {"tokens": 0}, {"tokens": (1 << 22) + 1}, {"cols": 0}, {"cols": 1 << 22}, {"ld_x": 49}, {"x": None}, {"x": ODD},
    {"stash": None}, {"stash": C.c_void_p((1 << 20) + 8)}, {"slots": 1 << 30, "tokens": 1000})]
CASES += [("tbp_stash8_get", GET, change) for change in ({"dtype": 2}, {"slot": 2}, {"tokens": 0}, {"ld_y": 49}, {"y": None}, {"y": ODD}, {"stash": None})]
CASES += [("tbp_stash8_dw", DW, change) for change in (
    {"slots": -1}, {"tokens": 0}, {"m": 0}, {"n_out": 0}, {"first": -1}, {"n": -1}, {"n": 4}, {"first": 3}, {"first": (1 << 31) - 1, "n": 1}, {"ld_dw": 59}, {"x": None}, {"dy": None}, {"dw": None}, {"dw": ODD},
    {"x": ODD})]


@pytest.mark.parametrize("name,good,change", CASES, ids=lambda v: v if isinstance(v, str) else ",".join(v) if len(v) < 4 else "")
def test_bad_arguments_are_refused(name, good, change):
    _refused(getattr(tbp.lib(), name)(*{**good, **change}.values()))


@pytest.mark.parametrize("name,good,change", [
    ("tbp_qk_norm", NORM, {"rows": 0}), ("tbp_qk_norm", NORM, {"n_heads": 0, "n_kv_heads": 0}), ("tbp_qk_norm_p1", NORM_P1, {"rows": 0}), ("tbp_qk_norm_append", APPEND, {"n_new": 0}),
    ("tbp_qk_norm_append", APPEND, {"batch": 0}), ("tbp_packed_attention_fwd", PACKED, {"rows": 0}), ("tbp_packed_attention_p1", PACKED_P1, {"rows": 0}),
    ("tbp_stash8_dw", DW, {"n": 0, "accumulate": 1})])
def test_empty_calls_do_nothing(name, good, change):
    assert getattr(tbp.lib(), name)(*{**good, **change}.values()) == 0


def test_sizes_that_callers_are_asked_for():
    L = tbp.lib()
    assert L.tbp_qk_norm_partial_rows(0, 4, 2, 64) == 0 == L.tbp_qk_norm_partial_rows(5, 0, 0, 64)
    assert L.tbp_qk_norm_partial_rows(1, 1, 0, 2) == 1 and L.tbp_qk_norm_partial_rows(1 << 22, 32, 8, 128) == 512
    assert L.tbp_stash8_bytes(1, 1, 1) == 2048 + 128 and L.tbp_stash8_bytes(3, 1025, 33) == 3 * (17 * 2 * 2048 + 2 * 64 * 4)
    assert L.tbp_stash8_bytes(0, 1, 1) == 0 == L.tbp_stash8_bytes(1, 0, 1)
    # (no more than the integers need, but for the padding: 1 byte for 2 of bf16)
    assert L.tbp_stash8_bytes(8, 4096, 11008) < 1.01 * 8 * 4096 * 11008
    for n, rows, h, kv, dh in ((5, 8192, 32, 8, 128), (61, 4096, 12, 4, 64), (1, 1, 1, 1, 64), (1000, 3, 4, 2, 128), (1, 1 << 22, 8, 1, 128), (0, 100, 2, 1, 64)):
        got = L.tbp_packed_attention_p1_scratch_bytes(n, rows, h, kv, dh)
        assert h * rows * 4 <= got < h * rows * 4 + (1 << 30)
    assert L.tbp_packed_attention_p1_scratch_bytes(1, 0, 4, 2, 64) == 0 == L.tbp_packed_attention_p1_scratch_bytes(1, 8, 3, 2, 64)


def _bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _stash(slots=2, tokens=6, cols=40):
    return tbp.Stash8(tokens, cols, slots, device="cpu")


def _good_calls():
    """One call of every operator, with arguments that fit: 6 tokens, 4 query heads on 2 key heads of 64."""
    table, g = torch.zeros((16, 32, 2)), _bf(64)
    heads = dict(gq=g, gk=g, n_heads=4, n_kv_heads=2, head_dim=64, eps=1e-5)
    attn = dict(n_heads=4, n_kv_heads=2, head_dim=64)
    return {
        "norm": (tbp.tbp_qk_norm, dict(qk=_bf(6, 384), **heads, table=table, positions=_i32(6), out=_bf(6, 384))),
        "norm_p1": (tbp.tbp_qk_norm_p1, dict(d_out=_bf(6, 384), qk=_bf(6, 384), **heads, table=table, positions=_i32(6), out=_bf(6, 384), partials=torch.zeros((tbp.lib().tbp_qk_norm_partial_rows(6, 4, 2, 64), 128)))),
        "append": (tbp.tbp_qk_norm_append, dict(qkv=_bf(6, 512), **heads, table=table, lengths=_i32(2), cache_k=_bf(2, 8, 128), cache_v=_bf(2, 8, 128), q_out=_bf(6, 256))),
        "packed_fwd": (tbp.tbp_packed_attention_fwd, dict(qkv=_bf(6, 512), starts=_i32(3), **attn, out=_bf(6, 256), lse=torch.zeros((4, 6)))),
        "packed_p1": (tbp.tbp_packed_attention_p1, dict(qkv=_bf(6, 512), out=_bf(6, 256), d_out=_bf(6, 256), lse=torch.zeros((4, 6)), starts=_i32(3), **attn, dqkv=_bf(6, 512),
                                                        scratch=torch.zeros(1 << 22, dtype=torch.uint8))),
        "put": (lambda x: _stash().put(0, x), dict(x=_bf(6, 40))),
        "get": (lambda out: _stash().get(0, out), dict(out=_bf(6, 40))),
        "dw": (tbp.tbp_stash8_dw, dict(x=_stash(), dy=_stash(cols=50), dw=torch.zeros((40, 50)))),
    }


@pytest.mark.parametrize("name", list(_good_calls()))
def test_tensors_of_the_host_are_refused(name):
    call, good = _good_calls()[name]
    with pytest.raises(TypeError, match="GPU"):
        call(**good)


def _beside(rows, columns, ld, dtype=torch.bfloat16):
    """A view of `columns` columns of an array of `ld`: its leading dimension would cover more."""
    return torch.zeros((rows, ld), dtype=dtype)[:, :columns]


@pytest.mark.parametrize("name,what,given", [
    ("norm", "qk", _beside(6, 320, 512)), ("norm", "out", _bf(5, 384)), ("norm", "out", _beside(6, 256, 512)), ("norm", "gq", _bf(63)), ("norm", "gk", torch.zeros(64)),
    ("norm", "positions", _i32(5)), ("norm_p1", "qk", _bf(6, 320)), ("norm_p1", "d_out", _bf(5, 384)), ("norm_p1", "out", _bf(6, 320)), ("norm_p1", "partials", torch.zeros((1, 64))),
    ("append", "qkv", _beside(6, 384, 512)), ("append", "q_out", _bf(2, 256)), ("append", "gk", _bf(128)), ("append", "lengths", _i32(2).long()),
    ("packed_fwd", "qkv", _beside(6, 448, 512)), ("packed_fwd", "out", _bf(5, 256)), ("packed_fwd", "lse", torch.zeros((4, 5))), ("packed_fwd", "starts", _i32(3).long()),
    ("packed_fwd", "starts", _i32(0)), ("packed_fwd", "starts", _i32(3, 1)), ("packed_p1", "dqkv", _bf(5, 512)), ("packed_p1", "d_out", _bf(6, 320)), ("packed_p1", "lse", torch.zeros((3, 6))),
    ("put", "x", _bf(6, 41)), ("put", "x", _bf(5, 40)), ("put", "x", _bf(40, 6).t()), ("get", "out", _bf(5, 40)), ("get", "out", _beside(6, 32, 40)),
    ("dw", "dw", torch.zeros((39, 50))), ("dw", "dw", _bf(40, 50)), ("dw", "dw", _beside(40, 48, 50, torch.float32))],
    ids=lambda v: v if isinstance(v, str) else "x".join(map(str, v.shape)))
def test_tensors_that_do_not_fit_are_refused(name, what, given):
    call, good = _good_calls()[name]
    with pytest.raises(TypeError, match=what):
        call(**{**good, what: given})


def test_other_bad_calls_are_refused():
    call, good = _good_calls()["norm"]
    with pytest.raises(ValueError, match="seq"):
        call(**{**good, "positions": None, "table": torch.zeros((5, 32, 2))})
    with pytest.raises(ValueError, match="table"):
        call(**{**good, "table": None})
    with pytest.raises(ValueError, match="seq"):
        call(**{**good, "positions": None, "seq": 0})
    call, good = _good_calls()["packed_p1"]
    need = tbp.lib().tbp_packed_attention_p1_scratch_bytes(2, 6, 4, 2, 64)
    for scratch in (torch.zeros(need - 1, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8).expand(need)):
        with pytest.raises((TypeError, ValueError), match="scratch"):
            call(**{**good, "scratch": scratch})
    with pytest.raises(ValueError, match="slots"):
        tbp.tbp_stash8_dw(_stash(2), _stash(3))
    with pytest.raises(ValueError, match="tokens"):
        tbp.tbp_stash8_dw(_stash(), _stash(tokens=7))
    with pytest.raises(ValueError, match="accumulate"):
        tbp.tbp_stash8_dw(_stash(), _stash(), accumulate=True)
    with pytest.raises(ValueError, match="stash"):
        tbp.Stash8(0, 4, device="cpu")
    with pytest.raises(ValueError, match="whole"):
        call, good = _good_calls()["append"]
        call(**{**good, "qkv": _bf(5, 512)})


def test_packed_attention_takes_no_more_blocks_than_a_launch_has_threads_for():
    """A launch has up to 512 threads for every (key head, 64 rows or sequence), counted in 32 bits."""
    assert tbp.lib().tbp_packed_attention_p1_scratch_bytes(3, 1 << 22, 64, 64, 64) == 0
    assert b"2^23" in tbp.lib().tbp_last_error()
    assert tbp.lib().tbp_packed_attention_p1_scratch_bytes(1 << 20, 1 << 20, 8, 8, 128) == 0
    assert tbp.lib().tbp_packed_attention_p1_scratch_bytes(3, 1 << 22, 32, 8, 128) > 0


@pytest.mark.parametrize("size", [{"slots": 0}, {"slots": -1}, {"tokens": 0}, {"cols": 1 << 22}, {"tokens": 1 << 22, "slots": 1 << 15}], ids=str)
def test_a_stash_that_cannot_be_says_why(size):
    """The text is this refusal's, not that of a failure before it."""
    _refused(tbp.lib().tbp_packed_attention_fwd(*{**PACKED, "head_dim": 96}.values()), "head_dim")
    with pytest.raises(ValueError, match="no stash of .*(slots|tokens)[^:]*(at least|above|too large)"):
        tbp.Stash8(**{"tokens": 5, "cols": 4, "slots": 1, **size}, device="cpu")


def test_how_a_weight_gradient_from_the_stash_runs():
    assert tbp.tbp_stash8_dw_plan(4096, 11008, 4096, 8) == (192, 1) and tbp.tbp_stash8_dw_plan(100, 50, 60, 0) == (128, 1)
    tile, shares = tbp.tbp_stash8_dw_plan(2048, 512, 512, 8)
    assert tile == 128 and shares > 1 and tbp.lib().tbp_stash8_dw_workspace_bytes(2048, 512, 512, 8) == shares * 512 * 512 * 4
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, -1), (1, 1 << 22, 1, 1)):
        with pytest.raises(tbp.TbpError):
            tbp.tbp_stash8_dw_plan(*bad)
    _refused(tbp.lib().tbp_stash8_dw_plan(1, 1, 1, 1, None, C.byref(C.c_int())), "null")


def test_heads_that_a_thread_of_the_norms_takes():
    per = tbp.lib().tbp_qk_norm_heads_per_thread
    assert per(BF16, 8192, 32, 8, 128) == 4 == per(F32, 1 << 22, 1, 0, 512) and per(BF16, 16, 32, 8, 128) == 1 == per(F32, 0, 4, 2, 64)
    assert per(BF16, -1, 4, 2, 64) == 0 == per(BF16, 4, 4, 2, 0) and per(7, 4, 4, 2, 64) == 0 == per(BF16, 4, 1 << 25, 2, 64) and per(F32, 4, 4, 2, 514) == 0


def test_how_packed_attention_runs():
    p = tbp.tbp_packed_attention_plan(1, 200, 32, 8, 128)
    assert (p.query_heads, p.key_shares, p.scores_ahead, p.queries_most_first, p.keys) == (2, 2, 0, 0, 64) and p.parts > 1
    p = tbp.tbp_packed_attention_plan(1000, 1 << 17, 6, 2, 64)
    assert (p.query_heads, p.key_shares, p.scores_ahead, p.queries_most_first, p.keys, p.parts, p.keys_most_first) == (1, 1, 0, 0, 64, 1, 0)
    with pytest.raises(tbp.TbpError, match="head_dim"):
        tbp.tbp_packed_attention_plan(1, 200, 32, 8, 96)
    _refused(tbp.lib().tbp_packed_attention_plan(1, 200, 32, 8, 128, None), "null")


def test_packed_attention_takes_the_order_that_measured_faster():
    order = lambda *size: (lambda p: (p.queries_most_first, p.keys_most_first))(tbp.tbp_packed_attention_plan(*size))
    # sequences, rows, heads, key heads, head_dim: 4 and more percent between the two, whether lengths are alike or far apart (queries), or both
    for size, queries in (((8, 8192, 16, 8, 128), 1), ((12, 8192, 16, 4, 128), 1), ((12, 32768, 8, 1, 128), 1), ((24, 32768, 8, 2, 64), 1), ((24, 8192, 32, 4, 128), 0), ((5, 4096, 32, 8, 128), 1), ((12, 8192, 32, 8, 128), 0), ((24, 8192, 32, 8, 128), 0), ((5, 4096, 64, 8, 128), 0),
                          ((8, 4096, 64, 16, 128), 0), ((8, 8192, 32, 8, 64), 1), ((8, 16384, 32, 8, 64), 1), ((32, 16384, 32, 8, 64), 0), ((24, 8192, 64, 16, 64), 0)):
        assert order(*size)[0] == queries, size
    for size, keys in (((8, 4096, 32, 8, 128), 1), ((16, 4000, 32, 8, 128), 1), ((64, 12800, 32, 8, 128), 1), ((6, 8192, 8, 8, 128), 1), ((64, 8192, 8, 8, 128), 0), ((16, 8192, 16, 16, 128), 0),
                       ((48, 8192, 32, 16, 128), 0), ((32, 8192, 32, 8, 64), 1), ((64, 16384, 16, 16, 64), 0)):
        assert order(*size)[1] == keys, size
