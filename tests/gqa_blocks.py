"""Values that show a lost or doubled block of keys, for the attention with grouped heads.

Random values average out over many keys, and so does what a missing block does to a row.  Here each block of 64
keys has one dim of its own per key/value head (as many blocks share a dim as there are D of them), in which its keys
hold 1 and its first and last keys 64: a row that sees it all with nearly equal weights loses 64 / 190 of what the block
gives to that dim with either of these keys, and all of it with the block.  A dim has the blocks b, b + D, ...: with n of
them a lost or doubled block moves it by about 1 / n, its first or last key by 0.34 / n, where the bound below is
under 0.02 of it (bf16 results; weights within a factor of two of each other): n up to 16 is 64 * 16 * 128 = 131,072
keys of 128 dims.

The bound is that of gqa_util, element by element, with the rounding u_p of a probability that the form of the launch
really makes: 32 rows of bf16 write a probability as two bf16 values, the upper half cut off and the rest (below 2^-7
of it, enlarged by 2^-20 of the whole) rounded by at most 2^-8 of itself: 2^-15 + 2^-20 altogether."""
import numpy as np

from gqa_util import U
from oracle.paged import attend

FINE = 2.0 ** -15 + 2.0 ** -20


def block_values(n, KV, D):
    v = np.zeros((n, KV, D))
    t = np.arange(n)
    for h in range(KV):
        v[t, h, (t // 64 + 7 * h) % D] = np.where((t % 64 == 0) | (t % 64 == 63), 64.0, 1.0)
    return v


def check_blocks(got, q, k, v, seen, u_p, u_o, what):
    """got [n, H, D] against the oracle; returns the largest share of the bound."""
    o, absum, mag = attend(q, k, v, seen)
    d = (q.shape[2] * 2.0 ** -23 + 16 * 2.0 ** -24) * mag[..., None] + 2.0 ** -21
    tol = absum * (2 * u_p + 2 * d + 2 * k.shape[0] * 2.0 ** -24) * 1.01 + np.abs(o) * u_o * 1.01 + 2.0 ** -40
    err = np.abs(got - o)
    worst = float((err / tol).max())
    at = np.unravel_index(np.argmax(err / tol), err.shape)
    assert worst <= 1.0, "%s: %.3g of the bound at row, head, dim %s: %r for %r" % (what, worst, at, got[at], o[at])
    return worst


def u_p(v_type, fine):
    return FINE if fine else (0.0 if v_type == "f32" else U[v_type])
