"""A paged cache that stays within a budget (oracle, plain Python and fp64).

The paper says nothing of positions or of what a long cache may lose.  Readings:

Rotary positions.  RoFormer's rotation (Su et al., 2021) of pairs of a head's
first R dims, half the turned dims apart or neighbours, with the frequencies
theta^(-2 j / R) or one of four forms stretched for long contexts: all by the
factor, a larger theta, by bands of wavelength, by a ramp over the pairs.

Attention weight.  What the softmax gives to a cached token, summed over rows
and the query heads that share its key/value head.

Eviction.  The tokens with the least weight go; the first and the most recent
ones stay.  Those behind the budget move into the places that are given up.
"""
import math

import numpy as np


def frequencies(R, theta, scaling="plain", factor=1.0, low=1.0, high=4.0, original=4096):
    """[R / 2] radians a position."""
    f = []
    for j in range(R // 2):
        t = theta * factor ** (R / (R - 2)) if scaling == "base" and R > 2 else theta
        g = t ** (-2.0 * j / R)
        if scaling == "linear":
            g /= factor
        elif scaling == "bands":
            turns = original * g / (2 * math.pi)
            if turns <= low:
                g /= factor
            elif turns < high:
                k = (turns - low) / (high - low)
                g = k * g + (1 - k) * g / factor
        elif scaling == "ramp":
            a, b = (R * math.log(original / (2 * math.pi * t)) / (2 * math.log(theta)) for t in (high, low))
            a, b = max(math.floor(a), 0), min(math.ceil(b), R - 1)
            k = 1.0 - min(1.0, max(0.0, (j - a) / (b - a if b > a else 0.001)))
            g = k * g + (1 - k) * g / factor
        f.append(g)
    return np.array(f)


def rotate(x, positions, freq, layout, inverse=False, magnitude=1.0):
    """x [n, heads, D]: pairs of the first 2 len(freq) dims turn by position * freq, "half" or "pairs"."""
    x = np.array(x, np.float64)
    R = 2 * len(freq)
    a = np.arange(R // 2) * (2 if layout == "pairs" else 1)
    b = a + (1 if layout == "pairs" else R // 2)
    t = np.asarray(positions, np.float64)[:, None] * freq
    c, s = magnitude * np.cos(t)[:, None], magnitude * np.sin(t)[:, None] * (-1 if inverse else 1)
    u, v = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = u * c - v * s, v * c + u * s
    return x


def weights(q, k, seen, scale=None):
    """q [n, H, D], k [L, KV, D], seen [n, L] -> (w [L, KV], and for an error bound of the same shape: sums of p_i
    times the largest scale * sum_d |q_d k_jd| of row i, and of p_i times the number of keys that it sees)."""
    n, H, D = q.shape
    L, KV = k.shape[:2]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    w, mag, keys = np.zeros((L, KV)), np.zeros((L, KV)), np.zeros((L, KV))
    for i in range(n):
        at = np.nonzero(seen[i])[0]
        if at.size == 0:
            continue
        for h in range(H):
            g = h // (H // KV)
            kk = k[at, g]
            s = scale * (kk @ q[i, h])
            p = np.exp(s - s.max())
            p /= p.sum()
            w[at, g] += p
            mag[at, g] += p * abs(scale) * (np.abs(kk) @ np.abs(q[i, h])).max()
            keys[at, g] += p * at.size
    return w, mag, keys


def choose(weight, number, N, first, recent, seen):
    """The places that stay, of one head's [L] weights and numbers: a list of N places, protected ones before
    the others, then the heavier (NaN above all), then the lower."""
    def worth(j):
        w = float(weight[j])
        kept = number[j] < first or number[j] >= seen - recent
        return (not kept, 0 if math.isnan(w) else 1, 0.0 if math.isnan(w) else -w, j)
    return sorted(range(len(weight)), key=worth)[:N]


def moves(stay, N):
    """(from, to) lists: the i-th place below N that is given up takes the i-th kept one from N on."""
    held = set(stay)
    return sorted(j for j in stay if j >= N), [j for j in range(N) if j not in held]
