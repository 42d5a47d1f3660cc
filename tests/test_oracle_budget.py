"""Pins of the oracle of a cache within a budget (no GPU): rotations by their invariants, frequencies at the ends of
their bands, weights as the attention's own probabilities, choices by brute force."""
import itertools
import math

import numpy as np
import pytest

from oracle.budget import choose, frequencies, moves, rotate, weights
from oracle.paged import attend
from oracle.rope import apply_rope

RNG = np.random.default_rng(5)


def test_plain_half_layout_is_the_layer_s():
    x, pos = RNG.standard_normal((5, 3, 16)), np.array([0, 1, 7, 100, 5000])
    want = apply_rope(x.reshape(5, -1), pos, 3, 10000.0).reshape(x.shape)
    assert np.allclose(rotate(x, pos, frequencies(16, 10000.0), "half"), want, rtol=0, atol=1e-12)


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("R", [2, 6, 16])
def test_rotations(layout, R):
    x, y = RNG.standard_normal((4, 2, 16)), RNG.standard_normal((4, 2, 16))
    f, pos = frequencies(R, 100.0), np.array([0, 3, 11, 64])
    r = rotate(x, pos, f, layout)
    assert np.allclose((r ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(r[..., R:], x[..., R:])
    assert np.allclose(rotate(r, pos, f, layout, inverse=True), x)
    assert np.array_equal(rotate(x, np.zeros(4), f, layout), x)
    # products depend on the distance alone
    a = (rotate(x, pos, f, layout) * rotate(y, pos + 5, f, layout)).sum(-1)
    b = (rotate(x, pos + 9, f, layout) * rotate(y, pos + 14, f, layout)).sum(-1)
    assert np.allclose(a, b)
    # the inverse is the transposed map, also with a magnitude
    a = (rotate(x, pos, f, layout, magnitude=1.3) * y).sum()
    b = (x * rotate(y, pos, f, layout, inverse=True, magnitude=1.3)).sum()
    assert np.isclose(a, b)


def test_pairs_turn_by_complex_numbers():
    x, pos, f = RNG.standard_normal((3, 1, 8)), np.array([2, 5, 9]), frequencies(8, 50.0)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * pos[:, None, None] * f)
    r = rotate(x, pos, f, "pairs")
    assert np.allclose(r[..., 0::2], z.real) and np.allclose(r[..., 1::2], z.imag)


def test_frequencies():
    assert np.allclose(frequencies(8, 10000.0), [1, 0.1, 0.01, 0.001])
    assert np.allclose(frequencies(8, 10000.0, "linear", 4.0), np.array([1, 0.1, 0.01, 0.001]) / 4)
    # a larger theta: the first pair stays, the last one is stretched by the whole factor
    f = frequencies(8, 10000.0, "base", 4.0)
    assert np.isclose(f[0], 1.0) and np.isclose(f[-1], 0.001 / 4)
    for kind in ("bands", "ramp"):
        plain = frequencies(64, 10000.0)
        f = frequencies(64, 10000.0, kind, 8.0, 1.0, 32.0 if kind == "ramp" else 4.0, 2048)
        assert np.isclose(f[0], plain[0]) and np.isclose(f[-1], plain[-1] / 8)
        ratio = f / plain
        assert (np.diff(ratio) <= 1e-12).all() and ((ratio > 0.13) & (ratio < 0.99)).any()
        assert np.allclose(frequencies(64, 10000.0, kind, 1.0, 1.0, 4.0, 2048), plain)
    # a pair of exactly the geometric middle: 2 turns of [1, 4]
    n = 2048
    theta = (n / (2 * math.pi * 2)) ** 2                   # pair 1 of R = 4 turns n f / 2 pi = 2 times
    f = frequencies(4, theta, "bands", 10.0, 1.0, 4.0, n)[1]
    assert np.isclose(f, theta ** -0.5 * (1 / 3 + 2 / 3 / 10))


def test_weights_are_the_attention_s():
    """Values that are unit vectors of the keys: the output is the row of probabilities."""
    n, H, KV, L, D = 5, 4, 2, 8, 8
    q, k = RNG.standard_normal((n, H, D)), RNG.standard_normal((L, KV, D))
    seen = RNG.random((n, L)) < 0.6
    seen[2] = False
    v = np.repeat(np.eye(L)[:, None, :], KV, axis=1)
    o, _, _ = attend(q, k, v, seen, 0.3)
    w, _, keys = weights(q, k, seen, 0.3)
    assert np.allclose(w, o.reshape(n, KV, 2, L).sum((0, 2)).T)
    assert np.isclose(w.sum(), H * seen.any(1).sum()) and (w >= 0).all()


@pytest.mark.parametrize("seed", range(8))
def test_choice_by_brute_force(seed):
    """Of all subsets, the one whose sorted worth is largest."""
    r = np.random.default_rng(seed)
    L, N = 7, int(r.integers(0, 8))
    w = r.choice([0.0, 1.0, 2.0, -1.0, np.inf], L)
    number = r.permutation(L)
    first, recent = int(r.integers(0, 3)), int(r.integers(0, 3))
    stay = choose(w, number, N, first, recent, L)

    def worth(j):
        return (number[j] < first or number[j] >= L - recent, w[j], -j)
    best = max((sorted((worth(j) for j in s), reverse=True), sorted(s)) for s in itertools.combinations(range(L), min(N, L)))
    assert sorted(stay) == best[1]
    source, hole = moves(stay, min(N, L))
    assert len(source) == len(hole) and all(h < N <= s for s, h in zip(source, hole))
    after = list(range(L))
    for s, h in zip(source, hole):
        after[h] = s
    assert sorted(after[:min(N, L)]) == sorted(stay)


def test_nan_is_heaviest():
    assert choose([1.0, float("nan"), float("inf")], [0, 1, 2], 2, 0, 0, 3) == [1, 2]
