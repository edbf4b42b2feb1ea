"""The oracle of the operators around packed documents against what it is not written from: differences, other forms, single values."""
import numpy as np
import pytest

from oracle import operators as ops
from oracle import packed as ref

RNG = np.random.default_rng(7)


@pytest.mark.parametrize("layout,dh,rot", [(0, 8, 8), (1, 8, 4), (0, 6, 2), (1, 10, 10), (0, 4, 0)])
def test_norm_gradients_are_those_of_differences(layout, dh, rot):
    H, KV, rows, eps = 3, 2, 4, 0.1
    x, dy = RNG.normal(size=(rows, (H + KV) * dh)), RNG.normal(size=(rows, (H + KV) * dh))
    gq, gk, ang = 1 + RNG.normal(size=dh) / 5, 1 + RNG.normal(size=dh) / 5, RNG.normal(size=(rows, rot // 2)) * 3
    f = lambda a, g, k: float((ref.qk_norm(a, g, k, H, KV, eps, ang, layout) * dy).sum())
    dx, dg = ref.qk_norm_p1(dy, x, gq, gk, H, KV, eps, ang, layout)
    h = 1e-6
    for _ in range(20):
        at = RNG.integers(rows), RNG.integers(x.shape[1])
        d = np.zeros_like(x)
        d[at] = h
        assert abs((f(x + d, gq, gk) - f(x - d, gq, gk)) / (2 * h) - dx[at]) < 1e-7
    for c in range(dh):
        d = np.zeros(dh)
        d[c] = h
        assert abs((f(x, gq + d, gk) - f(x, gq - d, gk)) / (2 * h) - dg[0, c]) < 1e-7
        assert abs((f(x, gq, gk + d) - f(x, gq, gk - d)) / (2 * h) - dg[1, c]) < 1e-7


def test_norms_have_length_one_and_rotations_keep_it():
    x = RNG.normal(size=(5, 3 * 16)) * 7
    y = ref.qk_norm(x, np.ones(16), np.ones(16), 2, 1, 0.0, RNG.normal(size=(5, 8)), 1).reshape(5, 3, 16)
    assert np.allclose((y * y).mean(axis=2), 1.0)


def test_packed_sequences_do_not_see_each_other():
    H, KV, dh, starts = 4, 2, 8, [0, 3, 3, 4, 11]
    qkv, do = RNG.normal(size=(13, (H + 2 * KV) * dh)), RNG.normal(size=(13, H * dh))
    out, lse = ref.packed_attention_fwd(qkv, starts, H, KV, dh)
    g = ref.packed_attention_p1(qkv, do, starts, H, KV, dh)
    assert not out[11:].any() and not g[11:].any() and np.all(np.isneginf(lse[:, 11:]))
    # one long sequence under a mask of blocks gives the same
    for h in range(H):
        q, k, v = ops._heads(qkv, slice(0, 11), h, H, KV, dh)
        s = q @ k.T / np.sqrt(dh)
        which = np.repeat(np.arange(4), np.diff(starts))
        s = np.where((which[:, None] == which) & np.tril(np.ones((11, 11), bool)), s, -np.inf)
        e = np.exp(s - s.max(axis=1, keepdims=True))
        assert np.allclose(e @ v / e.sum(axis=1, keepdims=True), out[:11, h * dh:(h + 1) * dh])
        assert np.allclose(np.log(np.exp(s).sum(axis=1)), lse[h, :11])
    moved = qkv.copy()
    moved[4:11] += 1.0
    assert np.array_equal(ref.packed_attention_fwd(moved, starts, H, KV, dh)[0][:4], out[:4])


def test_held_values():
    x = np.zeros((1030, 7))
    x[:, 0] = np.linspace(-127, 127, 1030).round()                # whole numbers in range: as they are
    x[5, 1], x[6, 1], x[7, 1] = 127.5, 1.0, 3.0                    # above 127: multiples of 2, halves to even
    x[0, 2], x[1029, 2] = 1.0, 1000.0                             # (another block)
    x[0, 3] = 1e-45                                               # below the smallest scale
    x[3, 4], x[1028, 4] = np.inf, 2.0
    x[2, 5], x[1, 5] = 2.5, 126.0                                 # halves to even
    x[2, 6] = np.nan
    y = ref.held(x)
    assert np.array_equal(y[:, 0], x[:, 0])
    assert list(y[5:8, 1]) == [128.0, 0.0, 4.0]
    assert y[0, 2] == 1.0 and y[1029, 2] == 1000.0 and y[1028, 4] == 2.0 and np.all(np.isnan(y[:1024, 4])) and y[1025, 4] == 0
    assert y[0, 3] == 0.0 and y[2, 5] == 2.0 and np.all(np.isnan(y[:1024, 6]))


def test_held_values_are_within_half_a_step():
    x = RNG.normal(size=(1500, 9)) * np.exp(3 * RNG.normal(size=9))
    y = ref.held(x)
    for t in (slice(0, 1024), slice(1024, 1500)):
        top = np.abs(x[t]).max(axis=0)
        step = 2.0 ** np.ceil(np.log2(top / 127))
        assert np.all(np.abs(x[t] - y[t]) <= step / 2) and np.all(step / 2 <= top / 127) and np.all(np.abs(y[t]) <= 127 * step)


def test_weight_gradients_of_a_set_are_the_sum_of_its_micro_batches():
    xs, dys = [RNG.normal(size=(70, 5)) for _ in range(3)], [RNG.normal(size=(70, 4)) for _ in range(3)]
    dw, size = ref.stash8_dw(xs, dys)
    plain = sum(x.T @ d for x, d in zip(xs, dys))
    assert np.abs(dw - plain).max() < 0.02 * np.abs(plain).max() + 0.3 and np.all(size >= np.abs(dw) - 1e-12)
    assert np.array_equal(dw, sum(ref.stash8_dw([x], [d])[0] for x, d in zip(xs, dys)))
