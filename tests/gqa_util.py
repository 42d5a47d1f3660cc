"""Shared by the tests of the attention with grouped heads: building a call on
the GPU and holding its output to the float64 oracle.

Error bound, element by element.  With p the exact probabilities and A = sum_j
p_j |v_j|, the computed output differs from the exact one by at most
  A (2 u_p + 2 d + 2 n 2^-24) + |o| u_o + 2^-40:
u_p the rounding of a probability to V's type (half a step: bf16 2^-8, fp16
2^-11, fp32 none) in the sum and in its divisor; u_o the output's rounding; n
2^-24 the fp32 sums over n keys; d the relative error of exp(s - m): the score
is a sum of D products in fp32, off by at most D 2^-23 scale sum |q k| whatever
the order, scaled and shifted with a few roundings of size |s| 2^-24 each (s and
the reference, at most 2 scale sum |q k| together, through up to eight roundings
in the splits), and the exponential is good to 2^-21.
"""
import numpy as np

from oracle.paged import attend

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def bound(o, absum, mag, n_keys, D, dtype, v_type):
    u_p = 0.0 if v_type == "f32" else U[v_type]
    d = (D * 2.0 ** -23 + 16 * 2.0 ** -24) * mag[..., None] + 2.0 ** -21
    return absum * (2 * u_p + 2 * d + 2 * n_keys * 2.0 ** -24) * 1.01 + np.abs(o) * U[dtype] * 1.01 + 2.0 ** -40


def check(got, q, k, v, seen, dtype, v_type, what, rows=None, scale=None):
    """got [n, H, D] against the oracle on rows (default all); returns the largest share of the bound."""
    rows = np.arange(q.shape[0]) if rows is None else np.asarray(rows)
    o, absum, mag = attend(q[rows], k, v, seen[rows], scale)
    with np.errstate(invalid="ignore"):
        tol = bound(o, absum, mag, k.shape[0], q.shape[2], dtype, v_type)
    g = got[rows]
    bad_kind = np.isfinite(o) != np.isfinite(g)
    assert not bad_kind.any(), "%s: finite in one only at %s" % (what, np.argwhere(bad_kind)[:3].tolist())
    fine = np.isfinite(o)
    same = (np.isnan(o) == np.isnan(g)) & (fine | np.isnan(o) | (o == g))
    assert same.all(), "%s: another infinity or NaN at %s" % (what, np.argwhere(~same)[:3].tolist())
    err = np.where(fine, np.abs(np.where(fine, g, 0) - np.where(fine, o, 0)), 0.0)
    tol = np.where(fine & np.isfinite(tol), tol, 1.0)
    worst = float((err / tol).max()) if err.size else 0.0
    at = np.unravel_index(np.argmax(err / tol), err.shape) if err.size else None
    assert worst <= 1.0, "%s: %.3g of the bound at row, head, dim %s: %r for %r" % (what, worst, at, g[at], o[at])
    return worst


TYPES = {"bf16": ("bf16", "bf16"), "v16": ("bf16", "f16"), "f32": ("f32", "f32")}


def torch_types(kind):
    import torch
    t = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
    return tuple(t[n] for n in TYPES[kind])


def desc(S, kind, H, KV, D, scale=0.0):
    return S.seer_attn_desc(H, KV, D, S.SEER_DTYPE_F32 if kind == "f32" else S.SEER_DTYPE_BF16,
                            S.SEER_ATTN_V_F16 if kind == "v16" else 0, scale)


def workspace(S, d, rows, batch, fill=0xff):
    """Every byte 0xff: a NaN wherever a float is read before it is written."""
    import torch
    return torch.full((max(S.seer_attn_workspace_bytes(d, rows, batch), 256),), fill, dtype=torch.uint8, device="cuda")


def words_of(bits, words):
    """Python ints -> [rows][words] int64 with the same 64-bit patterns."""
    out = np.zeros((len(bits), words), np.uint64)
    for i, m in enumerate(bits):
        for w in range(words):
            out[i, w] = (m >> 64 * w) & 0xffffffffffffffff
    return out.view(np.int64)
