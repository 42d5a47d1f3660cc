"""The three forms of the attention weights (bf16 tiles, bf16 with scores kept, fp32) on the cases where they could
differ; the rule that chooses, compiled for the host, says which form a call takes."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from test_dispatch import CXX, _ask
from test_gpu_attn_weights import Call, _bits

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(CXX is None, reason="no host C++ compiler")]
FORM = "int answer(const long long* v) { return v[5] ? 1 + weights_few(v[0], (int)v[1], (int)v[2], (int)v[3], v[4], true) : 0; }"


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


def form(tmp_path, c, last=0):
    """The form that a call takes: tiles, scores (kept) or f32."""
    H, KV, _ = c.shape
    rows = min(c.rows, last * c.B) if last else c.rows
    places = -(-c.W * c.page // 64) * 64
    return ("f32", "tiles", "scores")[_ask(tmp_path, FORM, [(rows, c.B, H, KV, places, c.kind != "f32")])[0]]


# rows that the call allows for behind its own, in each form
PADS = [("bf16", "scores", 2), ("bf16", "tiles", 400), ("f32", "f32", 2)]


@pytest.mark.parametrize("mask", ["causal", "tree"])
@pytest.mark.parametrize("kind,want,pad", PADS)
def test_rows_of_nan(S, tmp_path, kind, want, pad, mask):
    """A row of NaN makes the weights of the keys that it sees NaN, and those of no other key; a key that it sees with a
    score of -inf is one of them, and one that only other rows see, with -inf, gets nothing."""
    lens, past = [6, 5], [70, 20]
    bits = [0b1, 0b11, 0b101, 0b1001, 0b10001, 0b100001, 0b1, 0b11, 0b101, 0b1101, 0b11001] if mask == "tree" else None
    c = Call(S, kind, 4, 2, 64, past, lens, pad=pad, bits=bits)
    assert form(tmp_path, c) == want
    c.q.copy_(c.q.abs())                               # so that a key of -inf has the score -inf, not NaN

    def key(b, j):
        return c.pool[c.table[b, j // 16], 0, :, j % 16]

    key(0, 9).fill_(float("-inf"))                     # seen by all rows
    key(0, 75).fill_(float("-inf"))                    # the last row's own
    c.run(mask)
    clean = host(c.weight)
    c.q[2] = float("nan")                              # sees 0 .. 69, and of the call's rows 0 .. 2, or 0 and 2
    c.weight.fill_(7.0)
    c.run(mask)
    got = host(c.weight)
    for j in range(76):
        seen = j < 70 or (j - 70 in (0, 1, 2) if mask == "causal" else j - 70 in (0, 2))
        w, before = got[c.table[0, j // 16], :, j % 16], clean[c.table[0, j // 16], :, j % 16]
        if seen:
            assert np.isnan(w).all(), "token %d" % j
        else:
            assert np.array_equal(w, before), "token %d: %r for %r" % (j, w, before)
    assert np.array_equal(clean[c.table[0, 4], :, 11], host(c.prev)[c.table[0, 4], :, 11]), "-inf gives nothing"
    for j in range(25):
        at = (c.table[1, j // 16], slice(None), j % 16)
        assert np.array_equal(got[at], clean[at]), "the other request, token %d" % j


@pytest.mark.parametrize("kind,want,H,KV,D,rows,keys", [("bf16", "tiles", 64, 16, 64, 4096, 8000), ("bf16", "tiles", 4, 1, 128, 4000, 600),
                                                        ("bf16", "scores", 4, 1, 128, 1000, 2100), ("f32", "f32", 8, 1, 4, 2000, 300)])
def test_many_equal_rows(S, tmp_path, kind, want, H, KV, D, rows, keys):
    """Thousands of equal probabilities: every key has n / keys, and the sum's error does not grow with n roundings to the
    same side.

    Bound, relative to n / keys: the logarithm of a row's sum, log2 keys < 13, is off by 2^-20 whatever the parts, so p by
    2^-20 and the exponential's 2^-21 (ln 2 below 1).  Of the sum's additions, each at most 2^-24: up to 32 within a tile of
    rows, one a tile, at most rows a lane / 64 tiles (scores: 8 and a / 8; fp32: 4 and a quarter of a / 16), a few to join
    lanes and parts."""
    import torch
    n = rows * (H // KV)
    fill = -(-n // 16) if want == "scores" else 1      # requests without rows, so that rows are few on average
    c = Call(S, kind, H, KV, D, [keys - rows] + [0] * (fill - 1), [rows] + [0] * (fill - 1), pad=0, page=64)
    assert form(tmp_path, c) == want
    c.pool[:, 0] = 0.0                                 # every score is 0
    c.run("none", prev=False)
    got = host(c.weight).transpose(0, 2, 1).reshape(-1, KV)
    at = np.array([int(c.table[0, j // 64]) * 64 + j % 64 for j in range(keys)])
    in_tile, tiles = {"tiles": (32, n // 64 + 1), "scores": (8, n // 8 + 1), "f32": (4, n // 64 + 1)}[want]
    tol = 2.0 ** -20 + 2.0 ** -21 + (in_tile + tiles + 24) * 2.0 ** -24
    err = np.abs(got[at] * keys / n - 1.0).max()
    log("  %s %d rows of %d: off by %.2e, bound %.2e" % (want, n, keys, err, tol))
    assert err <= tol


@pytest.mark.parametrize("mask", ["causal", "none", "tree"])
@pytest.mark.parametrize("H,KV,D", [(4, 2, 64), (7, 1, 128), (8, 8, 64)])
def test_tiles_with_pages_that_are_none(S, tmp_path, H, KV, D, mask):
    """Missing pages of 16 keys at each place of a tile of 64, whole tiles of them, the first and the last page of a
    request, before the call's rows and among them: seen by no row, written by none."""
    past, lens = [250, 64, 0, 33], [40, 70, 50, 3]
    for lost in ([0], [1], [2], [3], [4, 5, 6, 7], [0, 5, 10, 15, 17], [3, 4], [16, 18, 19]):
        for last in (0, 40) if len(lost) > 1 else (0,):
            c = Call(S, "bf16", H, KV, D, past, lens, bits=_bits(lens) if mask == "tree" else None)
            for b in range(c.B):
                held = -(-c.kv_len[b] // 16)
                for i, j in enumerate(lost):
                    c.table[b, j % held] = (-1, c.P, 1 << 30, -(1 << 31))[i % 4]
                if lost == [3, 4]:
                    c.table[b, held - 1] = -1
            c.table_d = dev(c.table)
            assert form(tmp_path, c, last) == "tiles"
            c.run(mask, last=last)
            c.check(mask, last=last)


def test_tiles_of_a_request_without_pages(S, tmp_path):
    """Every page missing: nothing is written, beside requests that have theirs."""
    for mask in ("causal", "none", "tree"):
        past, lens = [130, 70, 5], [50, 60, 70]
        c = Call(S, "bf16", 4, 2, 64, past, lens, bits=_bits(lens) if mask == "tree" else None)
        c.table[1, :] = -1
        c.table_d = dev(c.table)
        assert form(tmp_path, c) == "tiles"
        c.run(mask)
        c.check(mask)


@pytest.mark.parametrize("H,KV,D", [(4, 2, 64), (3, 3, 128), (16, 8, 64)])
def test_tiles_of_rows_that_see_nothing(S, tmp_path, H, KV, D):
    """Rows with empty bits, some and all of a tile; caches that are shorter than the call's rows, so that the first ones
    stand before the first key (causal), among them more than a tile of rows, and all but one."""
    lens = [70, 40, 90, 33]
    r = np.random.default_rng(1)
    some = [b if r.random() < 0.4 else 0 for b in _bits(lens)]
    for past, bits in (([0, 0, 0, 0], some), ([20, 0, 64, 1], some), ([0, 100, 0, 3], [0] * sum(lens))):
        c = Call(S, "bf16", H, KV, D, past, lens, bits=bits)
        assert form(tmp_path, c) == "tiles"
        c.run("tree")
        c.check("tree")
    for past in ([-3, -39, -70, 0], [-69, -1, -89, -32], [-64, 5, -65, -31]):
        c = Call(S, "bf16", H, KV, D, past, lens, pad=90)
        assert form(tmp_path, c) == "tiles"
        for mask in ("causal", "none"):
            c.run(mask)
            c.check(mask)
        assert form(tmp_path, c, 60) == "tiles"
        c.run("causal", last=60)
        c.check("causal", last=60)


@pytest.mark.parametrize("B", [129, 300])
@pytest.mark.parametrize("H,KV,D,lens", [(8, 1, 64, (0, 12)), (2, 2, 128, (10, 40)), (8, 8, 64, (10, 40))])
def test_tiles_of_many_requests(S, tmp_path, B, H, KV, D, lens):
    """More requests than are kept beside the line, and more than threads: ragged, some without rows."""
    r = np.random.default_rng(B)
    n = [int(x) for x in r.integers(*lens, B)]
    past = [int(x) for x in r.integers(0, 90, B)]
    for mask in ("causal", "tree"):
        c = Call(S, "bf16", H, KV, D, past, n, bits=_bits(n) if mask == "tree" else None)
        assert form(tmp_path, c) == "tiles"
        c.run(mask, decay=0.5)
        c.check(mask, decay=0.5, requests=set(range(0, B, 13)) | {B - 1})


def test_tiles_of_most_requests(S, tmp_path):
    """As many requests as a call takes, with rows enough for tiles, most in one of them: the line is at its longest beside
    the tiles and the logarithms."""
    r = np.random.default_rng(9)
    lens = [int(x) for x in r.integers(0, 3, 4096)]
    lens[77] = 400
    past = [int(x) for x in r.integers(0, 20, 4096)]
    c = Call(S, "bf16", 16, 1, 128, past, lens)
    assert form(tmp_path, c) == "tiles"
    c.run("causal")
    c.check("causal", requests=set(range(0, 4096, 61)) | {77})


def test_tiles_in_parts_of_many_requests(S, tmp_path):
    """Rows cut in parts for more than 128 requests: the launch that joins them finds its line by itself."""
    B = 140
    lens = [28] * B
    lens[0], lens[139] = 200, 120
    c = Call(S, "bf16", 16, 1, 64, [int(x) for x in np.random.default_rng(2).integers(0, 20, B)], lens, page=64)
    assert form(tmp_path, c) == "tiles"
    body = "int answer(const long long* v) { return weights_sums(v[0], (int)v[1], (int)v[2], (int)v[3], v[4]); }"
    places = -(-c.W * c.page // 64) * 64
    assert _ask(tmp_path, body, [(c.rows, B, 16, 1, places)])[0] > 1
    c.run("causal")
    c.check("causal", requests={0, 5, 138, 139})
