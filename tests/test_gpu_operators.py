"""GPU parity of the operators for long contexts, the last stage and serving against the oracle in 64 bits.

Tolerances, from the arithmetic: attention outputs as for the fused attention (bf16 operands of the second product and one rounding of
the result: 1e-2 of the largest element forward, 1.5e-2 backward, the row log-sum-exp 1e-5 relative to its size + 1 (fp32 sums)); a result
that is rounded once to bf16 2^-8 of the element; fp32 results of sums in fp32 2e-5 of the tensor's largest element."""
import numpy as np
import pytest
import torch

import paper_2405_18047_amd as tbp
import seeded_inputs as si
from gpu_util import DEV, max_rel, to_dev, to_np
from oracle import operators as ref

pytestmark = pytest.mark.gpu

NAN = float("nan")


def _rnd(seed, name, shape, dtype, scale=1.0):
    return si.store_round(scale * si.standard_normal(seed, name, shape), dtype)


def _say(msg):
    print(msg, flush=True)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _same_infinities(got, want):
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)) and np.array_equal(got[~fine], want[~fine])
    return fine


# ------------------------------------------------------------------------------------------- sliding-window attention
WINDOW_CASES = [  # seq, batch, H, KV, dh, window, sinks, lengths
    (1, 1, 1, 1, 64, 1, 0, None), (1, 3, 4, 2, 128, 5, 2, [1, 0, 1]), (2, 1, 2, 1, 128, 1, 0, None),
    (37, 2, 3, 1, 64, 1, 0, None), (64, 1, 2, 2, 128, 64, 0, None), (65, 1, 4, 2, 64, 31, 1, [65]),
    (129, 2, 2, 1, 128, 32, 3, [129, 64]), (131, 3, 6, 2, 64, 7, 0, [131, 0, 5]), (257, 1, 8, 2, 128, 100, 64, None),
    (300, 2, 4, 4, 64, 300, 0, [299, 1]), (333, 1, 5, 1, 128, 65, 129, None), (513, 1, 4, 2, 128, 1, 1, None),
    (700, 1, 3, 3, 64, 128, 200, [641]), (1001, 2, 4, 2, 128, 250, 4, [1001, 777]), (1100, 1, 8, 8, 64, 5000, 9, None),
    (1500, 1, 2, 1, 128, 200, 1500, None), (2500, 1, 3, 1, 64, 333, 130, None), (3000, 1, 4, 2, 64, 3, 3000, None), (2049, 1, 1, 1, 128, 10, 700, [2048]),
    (90, 65, 8, 2, 64, 20, 2, None), (140, 40, 4, 4, 128, 50, 1, [140 - 3 * i for i in range(40)]), (600, 5, 16, 4, 128, 90, 5, None),
    (1100, 4, 16, 8, 128, 800, 5, [1100, 1037, 3, 900]), (1090, 2, 16, 16, 128, 900, 140, None), (1030, 4, 16, 4, 64, 800, 70, [1030, 1029, 0, 600]),
]


def _window_inputs(case, seed):
    seq, nb, H, KV, dh, _, _, lengths = case
    qkv, do = _rnd(seed, "qkv", (nb * seq, (H + 2 * KV) * dh), "bf16"), _rnd(seed, "do", (nb * seq, H * dh), "bf16")
    dev = to_dev(qkv, "bf16"), to_dev(do, "bf16")
    for b, n in enumerate(lengths or []):                       # what lies behind a sequence must not matter
        dev[0][b * seq + n:(b + 1) * seq] = NAN
        dev[1][b * seq + n:(b + 1) * seq] = NAN
    return qkv.astype(np.float64), do.astype(np.float64), *dev


@pytest.mark.parametrize("case", WINDOW_CASES, ids=str)
def test_window_attention_matches_oracle(case):
    seq, nb, H, KV, dh, window, sinks, lengths = case
    _say(f"window attention {case}")
    qkv, do, dqkv_in, ddo = _window_inputs(case, 61)
    o_ref, lse_ref = ref.window_attention_fwd(qkv, seq, H, KV, dh, window, sinks, lengths)
    g_ref = ref.window_attention_p1(qkv, do, seq, H, KV, dh, window, sinks, lengths)
    n = None if lengths is None else _ints(lengths)
    out, lse = tbp.tbp_window_attention_fwd(dqkv_in, seq, H, KV, dh, window, sinks, n)
    got = tbp.tbp_window_attention_p1(dqkv_in, out, ddo, lse, seq, H, KV, dh, window, sinks, n)
    torch.cuda.synchronize()
    assert max_rel(to_np(out), o_ref) < 1e-2
    l = to_np(lse) * np.log(2.0)
    fine = _same_infinities(l, lse_ref)
    assert np.all(np.abs(l - lse_ref)[fine] < 1e-5 * (1 + np.abs(lse_ref[fine])))
    got = to_np(got)
    assert np.all(np.isfinite(got))
    at = 0
    for name, width in (("dq", H * dh), ("dk", KV * dh), ("dv", KV * dh)):
        r, g = g_ref[:, at:at + width], got[:, at:at + width]
        at += width
        # (where every query sees one key, dq and dk are zero: what is left is the rounding of dP - delta, in units of dv's inputs)
        err = np.max(np.abs(g - r)) / max(np.max(np.abs(r)), 0.25)
        _say(f"   {name}: {err:.2e}")
        assert err < 1.5e-2, name
    for b, m in enumerate(lengths or []):
        assert not np.any(got[b * seq + m:(b + 1) * seq]) and not np.any(to_np(out)[b * seq + m:(b + 1) * seq])


def _row_errors(qkv, do, seq, H, KV, dh, window, sinks, lengths=None):
    """The oracle's out | dq | dk | dv with, for every row of every head of each, the error (a norm over the head's columns) that the arithmetic allows.

    A probability or score gradient rounded to bf16 is off by sigma = 2^-8 / sqrt 3 of itself at most, as a root mean square, in random directions: a row that
    adds n of them up with weights w and vectors x is off by sigma sqrt(sum w^2 |x|^2).  The output's error (P rounded, then the result: sigma sqrt 2 of
    it) reaches delta = do . o, and by dS = P (dP - delta) dq and dk.  Six times that, one rounding of the result, and 1e-3 for fp32 (dP - delta of
    a row that sees one key, lse)."""
    sigma, nb, G = 2.0 ** -8 / 3 ** 0.5, len(qkv) // seq, H // KV
    want = [ref.window_attention_fwd(qkv, seq, H, KV, dh, window, sinks, lengths)[0]]
    g = ref.window_attention_p1(qkv, do, seq, H, KV, dh, window, sinks, lengths)
    want += [g[:, :H * dh], g[:, H * dh:(H + KV) * dh], g[:, (H + KV) * dh:]]
    off = [np.zeros((len(qkv), n)) for n in (H, H, KV, KV)]       # squares
    sq = lambda z: (z * z).sum(axis=1)
    for b in range(nb):
        n = ref._length(lengths, b, seq)
        rows = slice(b * seq, b * seq + n)
        for h in range(H if n else 0):
            q, k, v = ref._heads(qkv, rows, h, H, KV, dh)
            o, d = want[0][rows, h * dh:(h + 1) * dh], do[rows, h * dh:(h + 1) * dh]
            p, _ = ref._softmax(q, k, window, sinks)
            dp = d @ v.T
            ds, p2 = (p * (dp - (dp * p).sum(axis=1, keepdims=True))) ** 2, p * p
            o_err = p2 @ sq(v)                                   # (of the sum; the result's own rounding is beside it)
            delta = (d * d * (o * o + o_err[:, None] / dh)).sum(axis=1) * 2
            off[0][rows, h] += o_err
            off[1][rows, h] += (ds @ sq(k) + delta * sq(p @ k)) / dh
            off[2][rows, h // G] += (ds.T @ sq(q) + p2.T @ (delta * sq(q))) / dh
            off[3][rows, h // G] += p2.T @ sq(d)
    size = [np.sqrt((w.reshape(len(qkv), -1, dh) ** 2).sum(axis=2)) for w in want]
    return want, [6 * sigma * np.sqrt(e) + 2.0 ** -8 * s + 1e-3 for e, s in zip(off, size)]


def _rows_fit(got, want, bounds, dh):
    """-> largest (error / bound) of the rows of out, dq, dk, dv."""
    return [float((np.sqrt(((a - w).reshape(len(w), -1, dh) ** 2).sum(axis=2)) / e).max()) for a, w, e in zip(got, want, bounds)]


@pytest.mark.parametrize("case", WINDOW_CASES, ids=str)
def test_window_attention_rows_are_right_to_their_own_size(case):
    """Late rows, whose sums of many small terms are small, are held to that, not to the largest element of all."""
    seq, nb, H, KV, dh, window, sinks, lengths = case
    _say(f"window attention row by row {case}")
    qkv, do, a, ddo = _window_inputs(case, 61)
    want, bounds = _row_errors(qkv, do, seq, H, KV, dh, window, sinks, lengths)
    n = None if lengths is None else _ints(lengths)
    out, lse = tbp.tbp_window_attention_fwd(a, seq, H, KV, dh, window, sinks, n)
    g = tbp.tbp_window_attention_p1(a, out, ddo, lse, seq, H, KV, dh, window, sinks, n)
    again = tbp.tbp_window_attention_fwd(a, seq, H, KV, dh, window, sinks, n)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])           # and the same every time
    assert torch.equal(g, tbp.tbp_window_attention_p1(a, out, ddo, lse, seq, H, KV, dh, window, sinks, n))
    g = to_np(g)
    fit = _rows_fit([to_np(out), g[:, :H * dh], g[:, H * dh:(H + KV) * dh], g[:, (H + KV) * dh:]], want, bounds, dh)
    _say("   largest error over its bound: " + ", ".join(f"{n} {f:.2f}" for n, f in zip(("out", "dq", "dk", "dv"), fit)))
    assert max(fit) < 1


def test_window_attention_with_wide_rows_keeps_what_is_beside_them():
    seq, nb, H, KV, dh, window, sinks = 203, 2, 4, 2, 64, 40, 3
    _say("window attention, wide rows")
    case = (seq, nb, H, KV, dh, window, sinks, None)
    qkv, do, a, ddo = _window_inputs(case, 62)
    w, wo = (H + 2 * KV) * dh, H * dh
    wide = torch.full((nb * seq, w + 24), NAN, dtype=torch.bfloat16, device=DEV)
    wide[:, 8:8 + w] = a
    out, dwide = torch.full((nb * seq, wo + 8), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((nb * seq, w + 16), 7.0, dtype=torch.bfloat16, device=DEV)
    dow = torch.full_like(out, NAN)
    dow[:, :wo] = ddo
    _, lse = tbp.tbp_window_attention_fwd(wide[:, 8:8 + w], seq, H, KV, dh, window, sinks, out=out[:, :wo])
    tbp.tbp_window_attention_p1(wide[:, 8:8 + w], out[:, :wo], dow[:, :wo], lse, seq, H, KV, dh, window, sinks, dqkv=dwide[:, 8:8 + w])
    plain, lse2 = tbp.tbp_window_attention_fwd(a, seq, H, KV, dh, window, sinks)
    g = tbp.tbp_window_attention_p1(a, plain, ddo, lse2, seq, H, KV, dh, window, sinks)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :wo], plain) and torch.equal(lse, lse2) and torch.equal(dwide[:, 8:8 + w], g)
    assert torch.all(out[:, wo:] == 7.0) and torch.all(dwide[:, :8] == 7.0) and torch.all(dwide[:, 8 + w:] == 7.0)


@pytest.mark.parametrize("seq,dh,window,sinks", [(300, 64, 40, 3), (1500, 128, 700, 0), (1500, 128, 100, 5)])
@pytest.mark.parametrize("bad", [NAN, float("inf")])
def test_window_attention_keeps_what_is_not_finite_within_its_sequence_and_key_head(seq, dh, window, sinks, bad):
    nb, H, KV = 6, 16, 8
    _say(f"window attention with {bad} seq={seq} dh={dh} window={window}")
    _, _, a, ddo = _window_inputs((seq, nb, H, KV, dh, window, sinks, None), 71)
    lengths = _ints([seq, seq, seq - 70, seq, seq, seq])
    run = lambda a: (lambda o, l: (o, l, tbp.tbp_window_attention_p1(a, o, ddo, l, seq, H, KV, dh, window, sinks, lengths)))(
        *tbp.tbp_window_attention_fwd(a, seq, H, KV, dh, window, sinks, lengths))
    clean = run(a)
    for column in (H + 3, H + KV + 3):                           # a key, then a value, of key head 3 of sequence 1
        dirty = a.clone()
        dirty[seq + 45, column * dh + 7] = bad
        got = run(dirty)
        ours = torch.zeros((nb, seq, H + 2 * KV), dtype=torch.bool, device=DEV)
        ours[1][:, [6, 7, H + 3, H + KV + 3]] = True             # its two query heads, the key head's derivatives
        same = lambda x, y, heads: bool((x == y).view(nb, seq, heads, dh).all(dim=3)[~ours[:, :, :heads]].all())
        assert same(got[0], clean[0], H) and same(got[2], clean[2], H + 2 * KV)
        assert bool((got[1] == clean[1]).transpose(1, 2)[~ours[:, :, :H]].all())
        if bad != bad or column == H + KV + 3:                   # (an infinite key may have a score of -infinity, which is a probability of zero)
            assert not bool(torch.isfinite(got[0].view(nb, seq, H, dh)[1, 45, 6:8]).all())


@pytest.mark.parametrize("gain", [8.0, 0.02])
@pytest.mark.parametrize("dh", [64, 128])
def test_window_attention_score_range(gain, dh):
    """Rows whose maximum climbs by many octaves, and rows where it hardly moves."""
    seq, H, KV, window, sinks = 640, 4, 2, 150, 5
    _say(f"window attention score range gain={gain} dh={dh}")
    qkv = _rnd(63, "qkv", (seq, (H + 2 * KV) * dh), "bf16")
    qkv[:, :H * dh] = si.round_bf16(qkv[:, :H * dh] * gain)
    o_ref, lse_ref = ref.window_attention_fwd(qkv.astype(np.float64), seq, H, KV, dh, window, sinks)
    out, lse = tbp.tbp_window_attention_fwd(to_dev(qkv, "bf16"), seq, H, KV, dh, window, sinks)
    assert max_rel(to_np(out), o_ref) < 1e-2
    assert np.max(np.abs(to_np(lse) * np.log(2.0) - lse_ref)) < 1e-5 * (1 + np.max(np.abs(lse_ref)))


def test_window_attention_gradient_against_differences():
    """dqkv along random directions against the change of the kernel's own outputs: dv exactly linear, dq and dk by the oracle's forward
    (a difference of bf16 outputs would be all rounding)."""
    seq, H, KV, dh, window, sinks = 70, 4, 2, 64, 20, 2
    _say("window attention, gradient against differences")
    case = (seq, 1, H, KV, dh, window, sinks, None)
    qkv, do, a, ddo = _window_inputs(case, 64)
    out, lse = tbp.tbp_window_attention_fwd(a, seq, H, KV, dh, window, sinks)
    g = to_np(tbp.tbp_window_attention_p1(a, out, ddo, lse, seq, H, KV, dh, window, sinks))
    for k in range(4):
        d = si.standard_normal(64, f"d{k}", qkv.shape)
        f = lambda z: float((ref.window_attention_fwd(z, seq, H, KV, dh, window, sinks)[0] * do).sum())
        want = (f(qkv + 1e-4 * d) - f(qkv - 1e-4 * d)) / 2e-4
        # errors of about 2^-9 of every element, of random sign, times a direction of unit variance
        assert abs(float((g * d).sum()) - want) < 6 * 4e-3 * np.sqrt((g * g).sum())


# ------------------------------------------------------------------------------------------- a token at a time over a cache
DECODE_CASES = [  # lengths, H, KV, dh, window, sinks, capacity
    ([1], 1, 1, 64, 1, 0, 1), ([0, 1, 2], 4, 2, 128, 3, 1, 8), ([5, 33, 64, 65], 8, 2, 128, 16, 4, 20), ([500], 32, 8, 128, 1024, 4, 1028),
    ([700, 31, 0, 1300], 12, 4, 64, 300, 3, 303), ([1000, 37], 40, 1, 128, 2000, 0, 1024), ([90] * 70, 6, 6, 64, 33, 2, 120),
    ([700 - 9 * i for i in range(50)], 16, 8, 128, 600, 4, 640), ([333, 0, 340] * 30, 8, 8, 64, 400, 0, 400), ([900] * 33, 8, 8, 128, 1000, 0, 901),
    ([3000, 2999], 8, 4, 128, 5000, 7, 1500), ([129, 128, 127], 35, 1, 64, 128, 0, 128), ([4, 3], 2, 1, 128, 10, 100, 101),
]


@pytest.mark.parametrize("case", DECODE_CASES, ids=str)
def test_window_decode_matches_oracle(case):
    lengths, H, KV, dh, window, sinks, capacity = case
    _say(f"window decode {case}")
    nb = len(lengths)
    q = _rnd(65, "q", (nb, H * dh), "bf16")
    o_ref, l_ref = np.zeros((nb, H * dh)), np.zeros((nb, H))
    ck, cv = (torch.full((nb, capacity, KV * dh), NAN, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for b, n in enumerate(lengths):
        k, v = (_rnd(65 + b, c, (n, KV * dh), "bf16") for c in ("k", "v"))
        o_ref[b], l_ref[b] = ref.window_decode(q[b].astype(np.float64), k.astype(np.float64), v.astype(np.float64), H, KV, dh, window, sinks, capacity)
        if n:
            p = np.array([i for i in range(n) if i < sinks or i >= n - (capacity - sinks)])
            rows = torch.tensor([ref.cache_row(int(i), capacity, sinks) for i in p], device=DEV)
            ck[b, rows], cv[b, rows] = to_dev(k[p], "bf16"), to_dev(v[p], "bf16")
    out, lse = tbp.tbp_window_decode(to_dev(q, "bf16"), ck, cv, _ints(lengths), H, KV, dh, window, sinks)
    torch.cuda.synchronize()
    assert max_rel(to_np(out), o_ref) < 1e-2
    l = to_np(lse) * np.log(2.0)
    fine = _same_infinities(l, l_ref)
    assert np.all(np.abs(l - l_ref)[fine] < 1e-5 * (1 + np.abs(l_ref[fine])))


def test_window_decode_calls_share_a_workspace():
    """Calls of one size after each other with one workspace, lengths from none to the whole window, so that the shares that a head's keys are cut
    into are many, few and one: each as with a workspace of its own."""
    nb, H, KV, dh, window, sinks = 3, 8, 2, 64, 4000, 4
    _say("decode calls with one workspace")
    ck, cv = (to_dev(_rnd(68, c, (nb * 4004, KV * dh), "bf16"), "bf16").view(nb, 4004, -1) for c in ("k", "v"))
    ws = tbp.tbp_window_decode_workspace(nb, H, KV, dh, window, sinks)
    assert ws is not None
    for i, lengths in enumerate(([4000, 1, 300], [0, 0, 0], [257, 256, 255], [9999, 5000, 4004], [700, 0, 31], [4004, 2000, 1000]) * 2):
        q = to_dev(_rnd(69 + i, "q", (nb, H * dh), "bf16"), "bf16")
        out, lse = tbp.tbp_window_decode(q, ck, cv, _ints(lengths), H, KV, dh, window, sinks, workspace=ws)
        o2, l2 = tbp.tbp_window_decode(q, ck, cv, _ints(lengths), H, KV, dh, window, sinks)
        assert torch.equal(out, o2) and torch.equal(lse, l2) and not bool(ws[:256].any())
        for b, n in enumerate(lengths):
            assert bool(torch.isfinite(lse[b]).all()) == (n > 0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_tokens_one_by_one_are_the_sequence_at_once(interleaved):
    """Appending and decoding token by token, over a ring that wraps, gives the rows of the rotation and forward of the whole sequence."""
    seq, nb, H, KV, dh, window, sinks, rot = 61, 3, 4, 2, 64, 13, 3, 32
    _say(f"token by token interleaved={interleaved}")
    layout = tbp.TBP_ROTARY_INTERLEAVED if interleaved else tbp.TBP_ROTARY_HALF
    qkv = to_dev(_rnd(66, "qkv", (nb * seq, (H + 2 * KV) * dh), "bf16"), "bf16")
    table = tbp.tbp_rotary_table(seq, rot, 10000.0)
    whole = qkv.clone()
    tbp.tbp_rotary(whole, H + KV, dh, table, seq=seq, layout=layout, out=whole)
    want, lse = tbp.tbp_window_attention_fwd(whole, seq, H, KV, dh, window, sinks)
    want, lse = to_np(want).reshape(nb, seq, -1), to_np(lse)
    ck, cv = (torch.full((nb, sinks + window, KV * dh), NAN, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    tokens = qkv.view(nb, seq, -1)
    t = 0
    for n in [7, 1, 20] + [1] * (seq - 28):                     # prompts of several tokens, longer than the ring, then single ones
        t += n
        lengths = _ints([t] * nb)
        q = tbp.tbp_rotary_append(tokens[:, t - n:t].reshape(nb * n, -1).contiguous(), H, KV, dh, table, lengths, ck, cv, sinks, layout=layout)
        out, l = tbp.tbp_window_decode(q.view(nb, n, -1)[:, -1].contiguous(), ck, cv, lengths, H, KV, dh, window, sinks)
        assert torch.equal(q, whole.view(nb, seq, -1)[:, t - n:t, :H * dh].reshape(nb * n, -1))
        assert np.max(np.abs(to_np(out) - want[:, t - 1])) < 2e-2 * np.max(np.abs(want[:, t - 1]))      # (two roundings of either)
        assert np.max(np.abs(to_np(l) - lse[:, :, t - 1])) < 1e-4


def test_decode_over_caches_whose_offsets_pass_32_bits():
    """A sequence whose cache spans more than 4 GiB: one wide array that the caches are columns of."""
    H, KV, dh, window, sinks, capacity, ld = 4, 1, 128, 64, 2, 700000, 4096
    _say("decode over 5.7 GB")
    base = torch.zeros((1, capacity, ld), dtype=torch.bfloat16, device=DEV)
    ck, cv = base[:, :, :dh], base[:, :, dh:2 * dh]
    n = capacity - 3
    k, v, q = (_rnd(67, c, (window + sinks, dh), "bf16") for c in ("k", "v", "q"))
    rows = torch.tensor(list(range(sinks)) + list(range(n - window, n)), device=DEV)
    base[0, rows, :dh], base[0, rows, dh:2 * dh] = to_dev(k, "bf16"), to_dev(v, "bf16")
    qq = q[:H].reshape(1, -1)
    o_ref, l_ref = ref.window_decode(qq[0].astype(np.float64), k.astype(np.float64), v.astype(np.float64), H, KV, dh, window, sinks, capacity)
    out, lse = tbp.tbp_window_decode(to_dev(qq, "bf16"), ck, cv, _ints([n]), H, KV, dh, window, sinks)
    assert max_rel(to_np(out)[0], o_ref) < 1e-2 and np.max(np.abs(to_np(lse)[0] * np.log(2.0) - l_ref)) < 1e-4
    # and the token's own rows are stored there
    table = tbp.tbp_rotary_table(capacity, dh, 10000.0)
    new = to_dev(_rnd(67, "new", (1, (H + 2 * KV) * dh), "bf16"), "bf16")
    tbp.tbp_rotary_append(new, H, KV, dh, table, _ints([n + 1]), ck, cv, sinks)
    assert torch.equal(base[0, n, dh:2 * dh], new[0, (H + KV) * dh:]) and bool((base[0, n, :dh] != 0).any())


# ------------------------------------------------------------------------------------------- rotary positions
ROTARY_CASES = [  # rows, seq, heads, dh, rot, ld, offset of the columns
    (1, 1, 1, 64, 64, 64, 0), (7, 7, 3, 128, 128, 400, 8), (50, 25, 5, 96, 32, 480, 0), (33, 11, 2, 64, 32, 132, 4),
    (19, 19, 3, 20, 12, 61, 1), (10, 5, 2, 6, 2, 14, 0), (2100, 700, 40, 128, 128, 5120, 0), (1000, 1000, 12, 64, 64, 2304, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", ROTARY_CASES, ids=str)
def test_rotary_matches_oracle(case, interleaved, dtype):
    rows, seq, heads, dh, rot, ld, off = case
    _say(f"rotary {case} interleaved={interleaved} {dtype}")
    layout = tbp.TBP_ROTARY_INTERLEAVED if interleaved else tbp.TBP_ROTARY_HALF
    n_pos, w = max(seq, 5000), heads * dh
    theta = ref.rotary_theta(rot, 10000.0)
    table = tbp.tbp_rotary_table(n_pos, rot, 10000.0)
    x = _rnd(71, "x", (rows, w), dtype)
    wide = torch.full((rows, ld + 8), 7.0, dtype=to_dev(x, dtype).dtype, device=DEV)
    wide[:, off:off + w] = to_dev(x, dtype)
    xin = wide[:, off:off + w]
    pos = np.random.default_rng(rows).integers(0, n_pos, rows)
    for positions, at in ((None, np.arange(rows) % seq), (_ints(pos.tolist()), pos)):
        for backward in (False, True):
            want = ref.rotary(x.astype(np.float64), heads, dh, theta, at, interleaved, backward)
            got = to_np(tbp.tbp_rotary(xin, heads, dh, table, positions, seq, layout, backward))
            # products of fp32 values of unit size, cosines good to 2^-24, then one rounding
            bound = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -22) * np.abs(want) + 1e-6 * np.max(np.abs(x))
            assert np.all(np.abs(got - want) <= bound)
    inplace = wide.clone()
    tbp.tbp_rotary(inplace[:, off:off + w], heads, dh, table, None, seq, layout, out=inplace[:, off:off + w])
    assert torch.equal(inplace[:, off:off + w], tbp.tbp_rotary(xin, heads, dh, table, None, seq, layout))
    assert torch.all(inplace[:, :off] == 7.0) and torch.all(inplace[:, off + w:] == 7.0)


def test_rotary_positions_outside_the_table_are_nan():
    table = tbp.tbp_rotary_table(16, 32, 10000.0)
    x = to_dev(_rnd(72, "x", (3, 128), "bf16"), "bf16")
    _say("rotary outside the table")
    y = to_np(tbp.tbp_rotary(x, 2, 64, table, _ints([3, 16, -1])))
    assert np.all(np.isfinite(y[0])) and np.all(np.isnan(y[1:].reshape(2, 2, 64)[:, :, :32]))
    assert np.array_equal(y[1:].reshape(2, 2, 64)[:, :, 32:], to_np(x)[1:].reshape(2, 2, 64)[:, :, 32:])


@pytest.mark.parametrize("name,kw", [("plain", {}), ("linear", {"factor": 4.0}), ("base", {"factor": 8.0}),
                                     ("ramp", {"factor": 16.0, "low": 1.0, "high": 32.0, "original": 4096.0})])
def test_rotary_tables(name, kw):
    """Angles of up to 100 000 turns of the fastest pair; cosines are rounded once to fp32."""
    _say(f"rotary table {name}")
    kind = {"plain": tbp.TBP_ROTARY_PLAIN, "linear": tbp.TBP_ROTARY_LINEAR, "base": tbp.TBP_ROTARY_BASE, "ramp": tbp.TBP_ROTARY_RAMP}[name]
    n_pos, rot = 100001, 24
    got = to_np(tbp.tbp_rotary_table(n_pos, rot, 10000.0, kind, magnitude=1.25, **kw))
    ang = np.arange(n_pos)[:, None] * ref.rotary_theta(rot, 10000.0, name, **kw)
    assert np.max(np.abs(got[..., 0] - 1.25 * np.cos(ang))) < 2e-7 and np.max(np.abs(got[..., 1] - 1.25 * np.sin(ang))) < 2e-7
    if name == "plain":                                          # the stage's own table, byte for byte
        assert torch.equal(tbp.tbp_rope_table(64, rot, 10000.0).view(torch.float32), tbp.tbp_rotary_table(64, rot, 10000.0).view(-1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_new,lengths,capacity,sinks", [(1, [1, 0, 9], 8, 2), (5, [5, 3, 40], 12, 4), (30, [30, 77, 0], 10, 0), (4, [4, 4, 4], 5, 4)])
def test_rotary_append_matches_oracle(dtype, n_new, lengths, capacity, sinks):
    H, KV, dh, rot = 4, 2, 32, 16
    _say(f"rotary append {dtype} n_new={n_new} lengths={lengths} capacity={capacity} sinks={sinks}")
    nb = len(lengths)
    x = _rnd(73, "x", (nb * n_new, (H + 2 * KV) * dh), dtype)
    ck, cv = (to_dev(_rnd(73, c, (nb * capacity, KV * dh), dtype), dtype).view(nb, capacity, -1) for c in ("ck", "cv"))
    k_ref, v_ref = to_np(ck), to_np(cv)
    table, theta = tbp.tbp_rotary_table(100, rot, 10000.0), ref.rotary_theta(rot, 10000.0)
    q = to_np(tbp.tbp_rotary_append(to_dev(x, dtype), H, KV, dh, table, _ints(lengths), ck, cv, sinks))
    tol = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -20
    for b, n in enumerate(lengths):
        for i in range(n_new):
            p, r = n - n_new + i, b * n_new + i
            if p < 0:
                assert not np.any(q[r])
                continue
            y = ref.rotary(x[r:r + 1].astype(np.float64), H + KV, dh, theta, [p])[0]
            assert np.all(np.abs(q[r] - y[:H * dh]) <= tol * np.abs(y[:H * dh]) + 4e-6)
            at = ref.cache_row(p, capacity, sinks)
            k_ref[b, at], v_ref[b, at] = y[H * dh:], x[r, (H + KV) * dh:]
    assert np.all(np.abs(to_np(ck) - k_ref) <= tol * np.abs(k_ref) + 4e-6)
    assert np.array_equal(to_np(cv), v_ref)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,dh,rot,H,KV", [("bf16", 128, 128, 18, 3), ("bf16", 128, 64, 9, 3), ("f32", 64, 64, 13, 1), ("bf16", 20, 12, 25, 5)])
def test_rotary_append_of_many_tokens(dtype, dh, rot, H, KV, interleaved):
    """Enough of them that a thread has four heads, of which q, k and v may be some: as rotating all of the rows by themselves (products of
    fp32 that may be contracted otherwise, one rounding of either)."""
    nb, n_new, capacity, sinks = 64, 200 if dh > 64 else 700, 150, 4
    assert nb * n_new * ((H + 2 * KV + 3) // 4) * (dh // 8) >= 4 * 256 * 256
    _say(f"rotary append of many tokens {dtype} dh={dh} rot={rot} H={H} KV={KV} interleaved={interleaved}")
    layout = tbp.TBP_ROTARY_INTERLEAVED if interleaved else tbp.TBP_ROTARY_HALF
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device=DEV)
    gen.manual_seed(74)
    qkv = torch.randn((nb * n_new, (H + 2 * KV) * dh), generator=gen, device=DEV).to(t)
    lengths = [n_new + 37 * b if b % 5 else n_new - 3 * b for b in range(nb)]
    table = tbp.tbp_rotary_table(4000, rot, 10000.0)
    ck, cv = (torch.full((nb, capacity, KV * dh), 7.0, device=DEV, dtype=t) for _ in range(2))
    q = tbp.tbp_rotary_append(qkv, H, KV, dh, table, _ints(lengths), ck, cv, sinks, layout=layout)
    pos = torch.tensor([[n - n_new + i for i in range(n_new)] for n in lengths], device=DEV)
    turned = tbp.tbp_rotary(qkv, H + KV, dh, table, pos.clamp(min=0).to(torch.int32).view(-1), layout=layout).view(nb, n_new, -1)
    want_q = torch.where(pos[..., None] >= 0, turned[..., :H * dh], torch.zeros((), device=DEV, dtype=t))
    near = lambda a, b: bool(((a.float() - b.float()).abs() <= (2.0 ** -7 if dtype == "bf16" else 2.0 ** -22) * b.float().abs() + 1e-5).all())
    assert near(q.view(nb, n_new, -1), want_q) and not bool(q.view(nb, n_new, -1)[pos < 0].any())
    v = qkv.view(nb, n_new, -1)[..., (H + KV) * dh:]
    want_k, want_v = torch.full_like(ck, 7.0), torch.full_like(cv, 7.0)
    for b, n in enumerate(lengths):
        new = [p for p in range(max(n - n_new, 0), n) if p < sinks or p >= n - (capacity - sinks)]
        rows, at = torch.tensor([ref.cache_row(p, capacity, sinks) for p in new], device=DEV), torch.tensor([p - (n - n_new) for p in new], device=DEV)
        want_k[b, rows], want_v[b, rows] = turned[b, at, H * dh:], v[b, at]
    assert near(ck, want_k) and torch.equal(ck == 7.0, want_k == 7.0) and torch.equal(cv, want_v)
    # and the rotation itself against the oracle, on some rows
    some = [0, 1, n_new * nb // 2, n_new * nb - 1]
    x, at = to_np(qkv[some]), pos.view(-1)[some].clamp(min=0).cpu().numpy()
    y = ref.rotary(x, H + KV, dh, ref.rotary_theta(rot, 10000.0), at, interleaved)
    assert np.all(np.abs(to_np(turned.reshape(nb * n_new, -1)[some]) - y) <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -22) * np.abs(y) + 1e-6 * np.max(np.abs(x)))


# ------------------------------------------------------------------------------------------- log probabilities
LOGIT_CASES = [(1, 1), (1, 2), (3, 7), (5, 63), (4, 64), (9, 1000), (2, 4097), (6, 50257), (1, 131072), (2, 200003), (300, 517), (700, 3001)]


def _logits(rows, vocab, dtype, seed=81):
    x = _rnd(seed, "x", (rows, vocab), dtype, 3.0)
    rng = np.random.default_rng([rows, vocab])
    t = rng.integers(-2, vocab + 2, rows)
    t[0] = vocab - 1
    if rows > 2 and vocab > 4:
        x[1, vocab // 2:] = -np.inf                              # masked columns, the target among them
        t[1] = vocab - 1
        x[2] = -np.inf                                           # nothing left
        t[2] = 1
    if rows > 4:
        x[3] = 1.5                                               # all alike
        x[4, ::2] = x[4, 0]                                      # many ties
    return x, t


def _logits_dev(x, dtype, pad, off):
    wide = torch.full((x.shape[0], x.shape[1] + pad), 100.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device=DEV)
    wide[:, off:off + x.shape[1]] = to_dev(x, dtype)
    return wide[:, off:off + x.shape[1]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,off", [(0, 0), (9, 5)])
@pytest.mark.parametrize("rows,vocab", LOGIT_CASES)
def test_logprobs_match_oracle(rows, vocab, dtype, pad, off):
    _say(f"logprobs rows={rows} vocab={vocab} {dtype} pad={pad}")
    x, t = _logits(rows, vocab, dtype)
    x64 = x.astype(np.float64)
    lp_ref, h_ref, lse_ref = ref.logprobs(x64, t)
    dev, tt = _logits_dev(x, dtype, pad, off), _ints(t.tolist())
    wl, wh = np.linspace(-1, 1, rows), np.linspace(0.5, -0.5, rows)
    fl, fh = (torch.tensor(v, dtype=torch.float32, device=DEV) for v in (wl, wh))
    g_ref = ref.logprobs_p1(x64, t, fl.double().cpu().numpy(), fh.double().cpu().numpy())
    for k in sorted({0, 1, min(5, vocab), min(64, vocab)}):
        got = tbp.tbp_logprobs(dev, tt, top=k)
        for a, r in zip(got[:3], (lp_ref, h_ref, lse_ref)):
            a = to_np(a)
            fine = _same_infinities(a, r)
            assert np.all(np.abs(a - r)[fine] <= 2e-5 * (1 + np.abs(r[fine])))
        if k:
            ids = got[4].cpu().numpy()
            for r in range(min(rows, 8)):
                want = ref.top(x[r], k) if vocab <= 5000 else list(np.lexsort((np.arange(vocab), -x64[r]))[:k])
                assert ids[r].tolist() == list(want), r
                v = to_np(got[3])[r]
                vr = x64[r, want] - lse_ref[r] if np.isfinite(lse_ref[r]) else np.full(k, -np.inf)
                fine = _same_infinities(v, vr)
                assert np.all(np.abs(v - vr)[fine] <= 2e-5 * (1 + np.abs(vr[fine])))
    logp, entropy, lse = got[:3]
    d1 = to_np(tbp.tbp_logprobs_p1(dev, tt, lse, entropy, fl, fh))
    s = tbp.tbp_logprobs_step(dev, tt, fl, fh)
    # p (1 + |log p| + H) |weight| with p good to 2^-20 or so, then one rounding
    bound = (2.0 ** -8 if dtype == "bf16" else 2e-5) * np.abs(g_ref) + 2e-5
    for d in (d1, to_np(s[3])):
        assert np.all(np.isfinite(d)) and np.all(np.abs(d - g_ref) <= bound)
    for a, r in zip(s[:3], (lp_ref, h_ref, lse_ref)):
        a = to_np(a)
        fine = _same_infinities(a, r)
        assert np.all(np.abs(a - r)[fine] <= 2e-5 * (1 + np.abs(r[fine])))


@pytest.mark.parametrize("rows,vocab", [(3, 50), (2, 40001)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logprobs_gradient_in_place_and_without_entropy(rows, vocab, dtype):
    _say(f"logprobs in place rows={rows} vocab={vocab} {dtype}")
    x, t = _logits(rows, vocab, dtype, 82)
    dev, tt = _logits_dev(x, dtype, 3, 1), _ints(t.tolist())
    w = torch.full((rows,), -0.5, device=DEV)
    _, h, lse = tbp.tbp_logprobs(dev, tt)
    want = tbp.tbp_logprobs_p1(dev, tt, lse, h, w)
    assert np.all(np.abs(to_np(want) - ref.logprobs_p1(x.astype(np.float64), t, [-0.5] * rows, [0.0] * rows)) <= 2.0 ** -8)
    a, b = _logits_dev(x, dtype, 3, 1), _logits_dev(x, dtype, 3, 1)
    tbp.tbp_logprobs_p1(a, tt, lse, h, w, out=a)
    tbp.tbp_logprobs_step(b, tt, w, out=b)
    assert torch.equal(a, want) and torch.equal(b, tbp.tbp_logprobs_step(dev, tt, w)[3])
    assert torch.all(a._base[:, 0] == 100.0) and torch.all(a._base[:, -2:] == 100.0) and torch.all(b._base[:, 0] == 100.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [50, 9000, 140000])
def test_logprobs_of_rows_masked_with_the_lowest_value(vocab, dtype):
    """Masked logits that are the type's lowest finite value: some of a row (probability zero), and all of it (the uniform distribution: entropy log
    vocab, to the fp32 sum of that many ones; lse, which has no room for log vocab beside it, is the lowest value)."""
    _say(f"logprobs, lowest values, vocab={vocab} {dtype}")
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    low = torch.finfo(t).min
    x = to_dev(_rnd(84, "x", (3, vocab), dtype), dtype)
    x[0, vocab // 2:] = low
    x[1] = low
    x[2, 1:] = low
    w, targets = torch.ones(3, device=DEV), _ints([0, 3, 0])
    logp, entropy, lse, top_logp, top_ids = tbp.tbp_logprobs(x, targets, top=5)
    s = tbp.tbp_logprobs_step(x, targets, w)
    half = ref.logprobs(to_np(x)[:1, :vocab // 2], [0])
    ln = float(np.log(vocab))
    for got in ((logp, entropy, lse), s[:3]):
        got = [to_np(g) for g in got]
        assert np.all(np.abs(np.array([g[0] for g in got]) - [h[0] for h in half]) <= 2e-5 * (1 + np.abs([h[0] for h in half])))
        assert abs(got[0][1] + ln) < 2e-5 * ln and abs(got[1][1] - ln) < 2e-5 * ln and got[2][1] == float(low)
        assert got[0][2] == 0.0 and got[1][2] == 0.0 and got[2][2] == float(x[2, 0])
    assert top_ids[1].tolist() == [0, 1, 2, 3, 4] and top_ids[2].tolist() == [0, 1, 2, 3, 4]
    assert np.all(np.abs(to_np(top_logp)[1] + ln) < 2e-5 * ln)
    d = to_np(s[3])
    want = np.full(vocab, -1.0 / vocab)
    want[3] += 1.0
    assert np.all(np.abs(d[1] - want) <= (2.0 ** -8 if dtype == "bf16" else 2e-5) * np.abs(want)) and not np.any(d[2])
    assert not np.any(d[0, vocab // 2:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [50, 9000, 140001])
@pytest.mark.parametrize("in_place", [False, True])
def test_logprobs_gradient_of_rows_whose_lse_does_not_show_the_sum(vocab, dtype, in_place):
    """The derivative by itself, from lse and entropy: rows of nothing but the type's lowest value (the uniform distribution), and rows of logits so large
    that a unit of lse's last place is 2^-9 and more; between them ordinary rows."""
    _say(f"logprobs gradient, large logits, vocab={vocab} {dtype} in place={in_place}")
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    x = _rnd(85, "x", (6, vocab), dtype, 3.0)
    x[1], x[2, 7:], x[2, :7] = low, low, low / 2
    x[3:5] = si.store_round(x[3:5] + np.array([[20000.0], [-300000.0]]), dtype)
    t, wl, wh = [0, 3, 2, vocab - 1, 1, -1], np.linspace(1, -1, 6).astype(np.float32), np.linspace(-0.5, 0.5, 6).astype(np.float32)
    g_ref = np.zeros((6, vocab))
    for r, row in enumerate(x.astype(np.float64)):               # (differences from the maximum first: 64 bits do not hold the sum beside the lowest value either)
        d = row - row.max()
        s = np.exp(d).sum()
        lp, p = d - np.log(s), np.exp(d) / s
        entropy = -(p * np.maximum(lp, -1e4)).sum()
        g_ref[r] = -p * (wl[r] if t[r] >= 0 else 0.0) - wh[r] * p * (np.maximum(lp, -1e4) + entropy)
        if t[r] >= 0:
            g_ref[r, t[r]] += wl[r]
    dev, tt, fl, fh = _logits_dev(x, dtype, 3, 1), _ints(t), torch.from_numpy(wl).to(DEV), torch.from_numpy(wh).to(DEV)
    _, entropy, lse = tbp.tbp_logprobs(dev, tt)
    got = to_np(tbp.tbp_logprobs_p1(dev, tt, lse, entropy, fl, fh, out=dev if in_place else None))
    # as in test_logprobs_match_oracle; ordinary rows have p from lse
    assert np.all(np.abs(got - g_ref) <= (2.0 ** -8 if dtype == "bf16" else 2e-5) * np.abs(g_ref) + 2e-5)
    assert torch.all(dev._base[:, 0] == 100.0) and torch.all(dev._base[:, -2:] == 100.0)


@pytest.mark.parametrize("bad", [NAN, float("inf")])
@pytest.mark.parametrize("vocab", [100, 70001])
def test_logprobs_of_rows_that_are_not_finite(bad, vocab):
    _say(f"logprobs with {bad} vocab={vocab}")
    x = to_dev(_rnd(83, "x", (3, vocab), "f32"), "f32")
    x[1, vocab // 3] = bad
    got = tbp.tbp_logprobs(x, _ints([0, 0, 0]), top=4)
    w = torch.ones(3, device=DEV)
    s = tbp.tbp_logprobs_step(x, _ints([0, 0, 0]), w, w)
    for a in list(got[:4]) + [s[3]]:
        a = to_np(a)
        assert np.all(np.isnan(a[1])) and np.all(np.isfinite(a[[0, 2]]))
    assert got[4][1].tolist() == [-1] * 4


# more rows than compute units: rows of every length at which another width of a row's threads is chosen, for the statistics, the ranking and the derivative
MANY_ROWS = [("bf16", 9001), ("bf16", 32000), ("bf16", 50257), ("bf16", 70001), ("f32", 3999), ("f32", 5003), ("f32", 16384), ("f32", 20011), ("f32", 40009),
             ("bf16", 8191), ("bf16", 2048)]


@pytest.mark.parametrize("dtype,vocab", MANY_ROWS)
def test_logprobs_of_many_rows_match_oracle(dtype, vocab):
    """As in test_logprobs_match_oracle, over more rows than compute units: every width of a row's threads; rows of padded and of even length."""
    rows = 259
    _say(f"logprobs of many rows vocab={vocab} {dtype}")
    x, t = _logits(rows, vocab, dtype, 86)
    some = [0, 1, 2, 3, 4, 100, 256, 257, 258]                   # (the oracle's rows; the others are compared between the calls)
    x64 = x[some].astype(np.float64)
    lp_ref, h_ref, lse_ref = ref.logprobs(x64, t[some])
    wl, wh = np.linspace(-1, 1, rows).astype(np.float32), np.linspace(0.5, -0.5, rows).astype(np.float32)
    g_ref = ref.logprobs_p1(x64, t[some], wl[some].astype(np.float64), wh[some].astype(np.float64))
    fl, fh = torch.from_numpy(wl).to(DEV), torch.from_numpy(wh).to(DEV)
    bound = (2.0 ** -8 if dtype == "bf16" else 2e-5) * np.abs(g_ref) + 2e-5
    for pad, off in ((0, 0), (9, 5)):
        dev, tt = _logits_dev(x, dtype, pad, off), _ints(t.tolist())
        got = {k: tbp.tbp_logprobs(dev, tt, top=k) for k in (0, 20, 64)}
        s = tbp.tbp_logprobs_step(dev, tt, fl, fh)
        for k, g in list(got.items()) + [(0, s)]:
            for a, r in zip(g[:3], (lp_ref, h_ref, lse_ref)):
                a = to_np(a)[some]
                fine = _same_infinities(a, r)
                assert np.all(np.abs(a[fine] - r[fine]) <= 2e-5 * (1 + np.abs(r[fine])))
            for a, b in zip(g[:3], got[0][:3]):                  # every row, whichever kernel it went through: to the order of the sums
                a, b = to_np(a), to_np(b)
                fine = _same_infinities(a, b)
                assert np.all(np.abs(a[fine] - b[fine]) <= 2e-5 * (1 + np.abs(b[fine])))
            if not k:
                continue
            ids, v = g[4].cpu().numpy(), to_np(g[3])
            for i, r in enumerate(some):
                want = np.lexsort((np.arange(vocab), -x64[i]))[:k]
                assert ids[r].tolist() == want.tolist(), (k, r)
                vr = x64[i, want] - lse_ref[i] if np.isfinite(lse_ref[i]) else np.full(k, -np.inf)
                fine = _same_infinities(v[r], vr)
                assert np.all(np.abs(v[r][fine] - vr[fine]) <= 2e-5 * (1 + np.abs(vr[fine])))
            order = torch.topk(dev.float(), k, dim=1).values     # (of every row: the values, which ties do not change)
            assert torch.equal(torch.gather(dev.float(), 1, g[4].long()), order)
        for d in (tbp.tbp_logprobs_p1(dev, tt, got[0][2], got[0][1], fl, fh), s[3]):
            assert np.all(np.abs(to_np(d[some]) - g_ref) <= bound) and bool(torch.isfinite(d).all())
        again = dev.clone()
        tbp.tbp_logprobs_step(again, tt, fl, fh, out=again)
        assert torch.equal(again, s[3])


@pytest.mark.parametrize("dtype,vocab", [("bf16", 1999), ("bf16", 2048), ("bf16", 5003), ("bf16", 8192), ("f32", 77), ("f32", 1024), ("f32", 3001)])
def test_logprobs_of_thousands_of_short_rows_match_oracle(dtype, vocab):
    """Rows that one wave takes, with and without the ranking and the derivative."""
    rows = 2101
    _say(f"logprobs of thousands of rows vocab={vocab} {dtype}")
    x, t = _logits(rows, vocab, dtype, 87)
    some = [0, 1, 2, 3, 4, 1000, 2047, 2048, 2100]
    x64 = x[some].astype(np.float64)
    refs = ref.logprobs(x64, t[some])
    wl, wh = np.linspace(-1, 1, rows).astype(np.float32), np.linspace(0.5, -0.5, rows).astype(np.float32)
    g_ref = ref.logprobs_p1(x64, t[some], wl[some].astype(np.float64), wh[some].astype(np.float64))
    dev, tt = _logits_dev(x, dtype, 9, 5), _ints(t.tolist())
    s = tbp.tbp_logprobs_step(dev, tt, torch.from_numpy(wl).to(DEV), torch.from_numpy(wh).to(DEV))
    for k in (0, 5, 32, 33):
        got = tbp.tbp_logprobs(dev, tt, top=k)
        for stats in (got, s):
            for a, r in zip(stats[:3], refs):
                a = to_np(a)[some]
                fine = _same_infinities(a, r)
                assert np.all(np.abs(a[fine] - r[fine]) <= 2e-5 * (1 + np.abs(r[fine])))
        if k:
            assert all(got[4][r].tolist() == np.lexsort((np.arange(vocab), -x64[i]))[:k].tolist() for i, r in enumerate(some))
            assert torch.equal(torch.gather(dev.float(), 1, got[4].long()), torch.topk(dev.float(), k, dim=1).values)
    assert np.all(np.abs(to_np(s[3][some]) - g_ref) <= (2.0 ** -8 if dtype == "bf16" else 2e-5) * np.abs(g_ref) + 2e-5)
    assert bool(torch.isfinite(s[3]).all())


def test_logprobs_of_as_many_rows_as_there_may_be():
    """2^31 - 1 rows of one logit each: the launches of a part of the rows each end behind the last one."""
    rows = 2 ** 31 - 1
    _say("logprobs of 2^31 - 1 rows")
    x = torch.empty((rows, 1), dtype=torch.bfloat16, device=DEV).normal_()
    targets, w = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.ones(rows, device=DEV)
    logp, entropy, lse = tbp.tbp_logprobs(x, targets)
    out = torch.full_like(x, NAN)
    tbp.tbp_logprobs_p1(x, targets, lse, entropy, w, out=out)
    for a, b, c, d, e in zip(*(t.view(-1).split(1 << 28) for t in (x, logp, entropy, lse, out))):
        assert torch.equal(d, a.float()) and not bool(b.any()) and not bool(c.any()) and not bool(e.any())
    del x, targets, w, logp, entropy, lse, out, a, b, c, d, e
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------- gradient norm and clipping
def _grads(sizes, dtype, scale=1.0):
    host = [_rnd(91, f"g{i}", (s,), dtype, scale) for i, s in enumerate(sizes)]
    return host, [to_dev(h, dtype) for h in host]


SIZES = [[1], [0, 5, 0], [8192], [8193, 8191, 7], [100003, 1, 64, 4096, 65536], [37] * 250, []]


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s or [0])}")
def test_grad_clip_matches_oracle(sizes, dtype, out):
    _say(f"grad clip {len(sizes)} tensors {dtype} -> {out}")
    host, dev = _grads(sizes, dtype)
    full = ref.grad_clip(host, 1e30)[0] if sizes else 0.0
    for max_norm in (0.5 * full, 2.0 * full + 1.0, 0.0):
        norm_ref, want = ref.grad_clip(host, max_norm)
        outs = [torch.full((s,), 7.0, dtype=torch.bfloat16 if out == "bf16" else torch.float32, device=DEV) for s in sizes]
        lst = tbp.GradList(dev, outs)
        norm = lst.clip(max_norm)
        sq = lst.sumsq()
        assert abs(float(norm) - norm_ref) <= 1e-6 * norm_ref and abs(float(sq) - norm_ref ** 2) <= 1e-12 * norm_ref ** 2
        for o, w in zip(outs, want):
            # the factor and the product in fp32, one rounding of the result
            assert np.all(np.abs(to_np(o) - w) <= (2.0 ** -8 if out == "bf16" else 2.0 ** -22) * np.abs(w))
        again = [torch.full_like(o, 3.0) for o in outs]
        tbp.GradList(dev, again).clip(max_norm, sumsq=sq)
        assert all(torch.equal(a, o) for a, o in zip(again, outs))


def test_grad_clip_in_place_of_unaligned_views_and_of_norms_that_are_not_finite():
    _say("grad clip in place, views, not finite")
    base = to_dev(_rnd(92, "b", (20011,), "f32"), "f32")
    for off in (0, 1, 3):
        g = base.clone()[off:]
        want = ref.grad_clip([to_np(g)], 1.0)
        lst = tbp.GradList([g])
        assert abs(float(lst.clip(1.0)) - want[0]) < 1e-6 * want[0]
        assert np.all(np.abs(to_np(g) - want[1][0]) <= 2.0 ** -22 * np.abs(want[1][0]))
        before = g.clone()
        lst.clip(2.0)
        assert torch.equal(g, before)
    for bad in (NAN, float("inf")):
        g = base.clone()
        g[777] = bad
        before = g.clone()
        norm = float(tbp.GradList([g]).clip(1.0))
        assert norm != norm if bad != bad else norm == float("inf")
        assert torch.equal(g.view(torch.int32), before.view(torch.int32))
    big = torch.full((3,), 3e38, device=DEV)                      # squares beyond fp32
    assert abs(float(tbp.GradList([big], [torch.empty_like(big)]).sumsq()) - 3 * float(big[0]) ** 2) < 1e-6 * 3 * float(big[0]) ** 2
    tbp.GradList([big]).clip(1.0)
    assert np.all(np.abs(to_np(big) - 1 / np.sqrt(3)) < 1e-6)


def _big_reference(tensors, max_norm):
    total = sum(float((t.double() ** 2).sum()) for t in tensors)
    return total, min(1.0, max_norm / total ** 0.5)


@pytest.mark.parametrize("sizes,dtype,out", [
    ([9_000_001, 3, 7_777_777, 1_000_003], "f32", "f32"),        # just above 16 M elements: pieces of 8192
    ([9_000_001, 3, 7_777_777, 1_000_003], "bf16", "bf16"),
    ([60_000_011, 45_000_017, 5], "f32", "bf16"),                # 420 MB: the norm reads past the caches; 6 pieces and more to a workgroup
    ([210_000_013, 100_003], "bf16", "f32"),
    ([10_000_019], "f32", "f32"),                                # pieces of 4096, several to a workgroup
], ids=lambda v: v if isinstance(v, str) else str(sum(v)))
def test_grad_clip_of_large_lists(sizes, dtype, out):
    """Sums of squares and clipped tensors against torch in 64 bits on the device, with a view that no piece of 16 bytes is aligned in among them."""
    _say(f"grad clip of {sum(sizes)} elements {dtype} -> {out}")
    gen = torch.Generator(device=DEV)
    gen.manual_seed(93)
    t, o = torch.bfloat16 if dtype == "bf16" else torch.float32, torch.bfloat16 if out == "bf16" else torch.float32
    grads = [torch.randn(s + 1, generator=gen, device=DEV, dtype=t)[1 if i % 2 else 0:][:s] for i, s in enumerate(sizes)]
    outs = [torch.full((s,), 7.0, dtype=o, device=DEV) for s in sizes]
    total, c = _big_reference(grads, 1.0)
    lst = tbp.GradList(grads, outs)
    norm, sq = lst.clip(1.0), lst.sumsq()
    # fp64 sums of this many squares: 1e-12 of the sum; the norm rounded to fp32; factor and product in fp32, one rounding of the result
    assert abs(float(sq) - total) <= 1e-12 * total and abs(float(norm) - total ** 0.5) <= 2.0 ** -23 * total ** 0.5
    for g, r in zip(grads, outs):
        want = g.double() * c
        assert bool(((r.double() - want).abs() <= (2.0 ** -8 if out == "bf16" else 2.0 ** -22) * want.abs()).all())
    if t is o:
        inplace = [g.clone() for g in grads]
        tbp.GradList(inplace).clip(1.0, sumsq=sq)
        assert all(torch.equal(a, b) for a, b in zip(inplace, outs))
    tbp.GradList(grads, outs).clip(2.0 * total ** 0.5)           # nothing to clip: passed on
    assert all(torch.equal(r, g.to(o)) for g, r in zip(grads, outs))


# ------------------------------------------------------------------------------------------- refusals
def test_one_tensor_of_the_host_among_a_call_s_is_refused():
    """The host refuses it; nothing is launched."""
    _say("tensors of the host")
    dev = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device=DEV)
    f, i = torch.float32, torch.int32
    table = dev(16, 32, 2, dtype=f)
    heads = dict(n_heads=4, n_kv_heads=2, head_dim=64)
    calls = [
        (tbp.tbp_window_attention_fwd, dict(qkv=dev(6, 512), seq=3, **heads, window=2, lengths=dev(2, dtype=i), out=dev(6, 256), lse=dev(2, 4, 3, dtype=f))),
        (tbp.tbp_window_attention_p1, dict(qkv=dev(6, 512), out=dev(6, 256), d_out=dev(6, 256), lse=dev(2, 4, 3, dtype=f), seq=3, **heads, window=2,
                                           lengths=dev(2, dtype=i), dqkv=dev(6, 512), scratch=dev(1 << 20, dtype=torch.uint8))),
        (tbp.tbp_window_decode, dict(q=dev(2, 256), cache_k=dev(2, 8, 128), cache_v=dev(2, 8, 128), lengths=dev(2, dtype=i), **heads, window=9000,
                                     out=dev(2, 256), lse=dev(2, 4, dtype=f), workspace=dev(1 << 22, dtype=torch.uint8))),
        (tbp.tbp_rotary, dict(x=dev(6, 384), n_heads=6, head_dim=64, table=table, positions=dev(6, dtype=i), out=dev(6, 384))),
        (tbp.tbp_rotary_append, dict(qkv=dev(6, 512), **heads, table=table, lengths=dev(2, dtype=i), cache_k=dev(2, 8, 128), cache_v=dev(2, 8, 128),
                                     q_out=dev(6, 256))),
        (tbp.tbp_logprobs, dict(logits=dev(6, 50), targets=dev(6, dtype=i))),
        (tbp.tbp_logprobs_p1, dict(logits=dev(6, 50), targets=dev(6, dtype=i), lse=dev(6, dtype=f), entropy=dev(6, dtype=f), d_logp=dev(6, dtype=f),
                                   d_entropy=dev(6, dtype=f), out=dev(6, 50))),
        (tbp.tbp_logprobs_step, dict(logits=dev(6, 50), targets=dev(6, dtype=i), d_logp=dev(6, dtype=f), d_entropy=dev(6, dtype=f), out=dev(6, 50))),
        (tbp.GradList([dev(8, dtype=f)]).clip, dict(max_norm=1.0, sumsq=dev(1, dtype=torch.float64), norm=dev(1, dtype=f))),
        (tbp.GradList([dev(8, dtype=f)]).sumsq, dict(out=dev(1, dtype=torch.float64))),
    ]
    for call, good in calls:
        call(**good)
        for k, v in good.items():
            if isinstance(v, torch.Tensor):
                with pytest.raises(TypeError, match="GPU"):
                    call(**{**good, k: v.cpu()})
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------- streams, graphs
def _everything(s):
    """One call of each operator into fixed outputs."""
    tbp.tbp_rotary(s["qkv"], 6, 64, s["table"], seq=200, out=s["rot"])
    s["rot_all"][:, :6 * 64].copy_(s["rot"])
    tbp.tbp_window_attention_fwd(s["rot_all"], 200, 4, 2, 64, 50, 3, out=s["out"], lse=s["lse"])
    tbp.tbp_window_attention_p1(s["rot_all"], s["out"], s["do"], s["lse"], 200, 4, 2, 64, 50, 3, dqkv=s["dqkv"], scratch=s["scratch"])
    tbp.tbp_rotary_append(s["qkv"][:2], 4, 2, 64, s["table"], s["lengths"], s["ck"], s["cv"], 3, q_out=s["q"])
    tbp.tbp_window_decode(s["q"], s["ck"], s["cv"], s["lengths"], 4, 2, 64, 50, 3, out=s["o1"], lse=s["l1"], workspace=s["ws"])
    s["top"] = tbp.tbp_logprobs(s["logits"], s["targets"], top=5)
    s["step"] = tbp.tbp_logprobs_step(s["logits"], s["targets"], s["w"])
    s["norm"] = s["list"].clip(1.0)


def _setup(seed):
    f = lambda n, *shape: to_dev(_rnd(seed, n, shape, "bf16"), "bf16")
    e = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device=DEV)
    L = tbp.lib()
    s = {"qkv": f("qkv", 400, 512), "do": f("do", 400, 256), "rot": e(400, 384), "out": e(400, 256), "lse": e(2, 4, 200, dtype=torch.float32),
         "dqkv": e(400, 512), "scratch": e(L.tbp_window_attention_p1_scratch_bytes(2, 4, 2, 200, 64, 50, 3), dtype=torch.uint8),
         "ck": f("ck", 2, 53, 128), "cv": f("cv", 2, 53, 128), "q": e(2, 256), "o1": e(2, 256), "l1": e(2, 4, dtype=torch.float32),
         "ws": tbp.tbp_window_decode_workspace(2, 4, 2, 64, 50, 3), "lengths": _ints([70, 20]), "table": tbp.tbp_rotary_table(200, 64, 1e4),
         "logits": f("logits", 5, 5000), "targets": _ints([1, 2, -1, 4, 5]), "w": torch.ones(5, device=DEV)}
    s["rot_all"] = s["qkv"].clone()
    g = [f("g", 3000).float(), f("g2", 17, 9).float()]
    s["list"] = tbp.GradList(g, [torch.empty_like(t) for t in g])
    return s


def _results(s):
    torch.cuda.synchronize()
    return [t.clone() for k in ("rot", "out", "lse", "dqkv", "ck", "cv", "q", "o1", "l1") for t in [s[k]]] + \
        [t.clone() for k in ("top", "step") for t in s[k]] + [s["norm"].clone()] + [t.clone() for t in s["list"].outs]


def test_operators_on_another_stream_give_the_same():
    _say("operators on another stream")
    a, b = _setup(101), _setup(101)
    _everything(a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _everything(b)
    assert all(torch.equal(x, y) for x, y in zip(_results(a), _results(b)))


def test_operators_replayed_from_a_graph_equal_the_eager_calls():
    _say("operators from a graph")
    s, other = _setup(102), _setup(103)
    want = []
    for src in (s, other):
        e = _setup(102)
        for k in ("qkv", "do", "rot_all", "ck", "cv", "logits"):
            e[k].copy_(src[k])
        _everything(e)
        want.append(_results(e))
    keep = {k: s[k].clone() for k in ("qkv", "do", "rot_all", "ck", "cv", "logits")}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _everything(s)
    for rep in range(4):
        for k in keep:
            s[k].copy_(keep[k] if rep % 2 == 0 else other[k] if k not in ("ck", "cv", "rot_all") else _setup(103)[k])
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(_results(s), want[rep % 2])), rep
        _everything(_setup(104))                                  # eager work between the replays
        torch.cuda.synchronize()
