"""Pins of the oracle of the operators for long contexts: derivatives against central differences, closed forms, and the
relations that tie one operator to another."""
import numpy as np
import pytest

from oracle import operators as ref


def _rng(*key):
    return np.random.default_rng(list(key))


def _difference(f, x, d, eps=1e-5):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


@pytest.mark.parametrize("window,sinks,lengths", [(3, 0, None), (3, 2, None), (20, 0, None), (1, 1, None), (2, 3, [7, 0])])
def test_window_attention_p1_is_the_derivative_of_the_forward(window, sinks, lengths):
    """Along random directions; central differences of a smooth function at 1e-5 are good to about 1e-9."""
    seq, H, KV, dh = 9, 4, 2, 6
    r = _rng(1, window, sinks)
    x, w, d = (r.standard_normal((2 * seq, c)) for c in ((H + 2 * KV) * dh, H * dh, (H + 2 * KV) * dh))
    f = lambda z: float((ref.window_attention_fwd(z, seq, H, KV, dh, window, sinks, lengths)[0] * w).sum())
    g = ref.window_attention_p1(x, w, seq, H, KV, dh, window, sinks, lengths)
    assert abs(_difference(f, x, d) - float((g * d).sum())) < 1e-7


def test_wide_window_is_causal_attention_and_sinks_are_its_first_keys():
    seq, H, dh = 11, 2, 4
    x = _rng(2).standard_normal((seq, 3 * H * dh))
    whole, _ = ref.window_attention_fwd(x, seq, H, H, dh, seq, 0)
    assert np.array_equal(whole, ref.window_attention_fwd(x, seq, H, H, dh, 1, seq)[0])
    assert np.array_equal(ref.window_attention_fwd(x, seq, H, H, dh, 1, 0)[0], x[:, 2 * H * dh:])        # every token sees itself alone
    from oracle import ops
    want, _ = ops.attention_fwd(x[:, :8], x[:, 8:16], x[:, 16:], seq, H, dh, True)
    assert np.max(np.abs(whole - want)) < 1e-13


def test_decode_is_the_forwards_last_row_and_a_ring_keeps_sinks_and_last_tokens():
    seq, H, KV, dh = 23, 4, 2, 4
    x = _rng(3).standard_normal((seq, (H + 2 * KV) * dh))
    for window, sinks in ((5, 0), (5, 3), (40, 2)):
        out, lse = ref.window_attention_fwd(x, seq, H, KV, dh, window, sinks)
        o, l = ref.window_decode(x[-1, :H * dh], x[:, H * dh:(H + KV) * dh], x[:, (H + KV) * dh:], H, KV, dh, window, sinks, sinks + max(window, seq))
        assert np.max(np.abs(o - out[-1])) < 1e-13 and np.max(np.abs(l - lse[0, :, -1])) < 1e-13
    held = {}
    for p in range(seq):
        held[ref.cache_row(p, 9, 3)] = p
    assert sorted(held.values()) == [0, 1, 2] + list(range(seq - 6, seq)) and sorted(held) == list(range(9))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_turns_pairs_and_its_derivative_is_the_transpose(interleaved):
    rows, heads, dh, rot = 5, 2, 10, 6
    r = _rng(4)
    x, d = r.standard_normal((rows, heads * dh)), r.standard_normal((rows, heads * dh))
    pos = [0, 3, 1000, 7, 7]
    for kw in ({}, {"scaling": "linear", "factor": 4.0}, {"scaling": "base", "factor": 4.0}, {"scaling": "ramp", "factor": 4.0, "original": 64.0, "high": 4.0}):
        theta = ref.rotary_theta(rot, 10000.0, **kw)
        y = ref.rotary(x, heads, dh, theta, pos, interleaved, magnitude=1.5)
        b = ref.rotary(d, heads, dh, theta, pos, interleaved, backward=True, magnitude=1.5)
        assert abs((y * d).sum() - (x * b).sum()) < 1e-11
        back = ref.rotary(ref.rotary(x, heads, dh, theta, pos, interleaved), heads, dh, theta, pos, interleaved, backward=True)
        assert np.max(np.abs(back - x)) < 1e-13
        # scores depend on the distance of positions alone
        q, k = x[:1], d[:1]
        s = [(ref.rotary(q, heads, dh, theta, [p + 5], interleaved) * ref.rotary(k, heads, dh, theta, [p], interleaved)).sum() for p in (0, 11)]
        assert abs(s[0] - s[1]) < 1e-12


def test_rotary_scalings_meet_their_ends():
    rot, base, f = 32, 10000.0, 8.0
    plain = ref.rotary_theta(rot, base)
    scaled = ref.rotary_theta(rot, base, "base", f)
    assert abs(scaled[0] - plain[0]) < 1e-15 and abs(scaled[-1] * f / plain[-1] - 1) < 1e-12
    ramp = ref.rotary_theta(rot, base, "ramp", f, 1.0, 32.0, 4096.0)
    turns = 4096.0 * plain / (2 * np.pi)
    assert np.array_equal(ramp[turns >= 32], plain[turns >= 32]) and np.max(np.abs(ramp[turns <= 1] * f / plain[turns <= 1] - 1)) < 1e-12
    assert np.all((ramp <= plain) & (ramp >= plain / f * (1 - 1e-12)))


def test_logprobs_p1_is_the_derivative_of_logp_and_entropy():
    rows, vocab = 4, 13
    r = _rng(5)
    x, d = 2 * r.standard_normal((rows, vocab)), r.standard_normal((rows, vocab))
    x[1, 5:] = -np.inf
    d[1, 5:] = 0.0
    t, wl, we = [3, 2, -1, 12], r.standard_normal(rows), r.standard_normal(rows)

    def f(z):
        logp, entropy, _ = ref.logprobs(z, t)
        return float(logp @ wl + entropy @ we)
    g = ref.logprobs_p1(x, t, wl, we)
    assert abs(_difference(f, x, d) - float((g * d).sum())) < 1e-7
    assert np.all(g[1, 5:] == 0.0) and np.max(np.abs(g.sum(axis=1))) < 1e-13        # (adding a constant changes nothing)
    logp, entropy, lse = ref.logprobs(np.full((1, 8), 0.25), [1])
    assert abs(logp[0] + np.log(8)) < 1e-15 and abs(entropy[0] - np.log(8)) < 1e-15 and abs(lse[0] - 0.25 - np.log(8)) < 1e-15
    logp, entropy, lse = ref.logprobs(np.full((1, 8), -np.inf), [1])
    assert logp[0] == -np.inf and lse[0] == -np.inf and entropy[0] == 0.0
    assert ref.top(np.array([1.0, 3.0, 3.0, -np.inf, 2.0]), 4) == [1, 2, 4, 0]


def test_grad_clip_scales_to_the_norm():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    norm, out = ref.grad_clip(g, 2.5)
    assert norm == 5.0 and np.array_equal(out[0], [1.5, 0.0]) and out[1][0, 0] == 2.0
    assert np.array_equal(ref.grad_clip(g, 5.0)[1][0], g[0])
    assert np.array_equal(ref.grad_clip([np.array([np.inf, 1.0])], 1.0)[1][0], [np.inf, 1.0])
