"""Pins for the oracle of paged keys and values (CPU only): the book-keeping
against hand values and against invariants over random steps, the attention
against torch's own float64 routine and against the packed computation."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle.paged import EXHAUSTED, INVALID, WIDTH, attend, cached_rows, pages_of, plan, sees


def test_plan_by_hand():
    table = [[7, 3, -1, -1], [5, 2, 9, -1], [-1, -1, -1, -1]]
    # request 0 grows from 20 to 33 + 1 tokens, request 1 keeps 16 of 40, request 2 starts with 17
    r = plan([20, 40, 0], [20, 16, 0], [14, 0, 18], [14, 0, 17], table, [0, 1, 4], 16, 10, 34)
    # given back: pages 2, 9 of request 1 -> stack 0 1 4 2 9; taken: 9 (request 0), 2, 4 (request 2)
    assert r["table"] == [[7, 3, 9, -1], [5, 2, 9, -1], [2, 4, -1, -1]]
    assert r["free"] == [0, 1] and r["kv_len"] == [34, 16, 17] and r["status"] == 0
    assert r["slots"] == list(range(3 * 16 + 4, 3 * 16 + 16)) + [9 * 16, 9 * 16 + 1] + list(range(32, 48)) + [64, -1] + [-1] * 2
    assert plan([20], [20], [40], None, [[1, 2]], [3, 4], 16, 5, 40)["status"] == WIDTH
    assert plan([20], [21], [1], None, [[1, 2]], [3, 4], 16, 5, 1)["status"] == INVALID
    assert plan([20], [20], [13], None, [[1, 2, -1]], [], 16, 5, 13)["status"] == EXHAUSTED
    assert plan([40], [0], [0], None, [[1, 2, 3]], [0, 4, 4], 16, 5, 0)["status"] == INVALID


def test_every_page_has_one_owner():
    rng = np.random.default_rng(3)
    B, W, P, page = 6, 5, 17, 16
    table, free, held = [[-1] * W for _ in range(B)], list(range(P)), [0] * B
    done = 0
    for _ in range(300):
        keep = [int(rng.integers(0, h + 1)) if rng.random() < 0.5 else h for h in held]
        lens = [int(rng.integers(0, 30)) for _ in range(B)]
        used = [int(rng.integers(0, n + 1)) for n in lens]
        r = plan(held, keep, lens, used, table, free, page, P, sum(lens))
        if r["status"]:
            assert (r["table"], r["free"], r["kv_len"]) == (table, free, held)
            held = r["kv_len"]
            keep = [0] * B                                       # end some requests
            r = plan(held, [h if b % 2 else 0 for b, h in enumerate(held)], [0] * B, None, table, free, page, P, 0)
            assert r["status"] == 0
        else:
            done += 1
            real = [s for s in r["slots"] if s >= 0]
            assert len(set(real)) == len(real) == sum(used)
        table, free, held = r["table"], r["free"], r["kv_len"]
        owned = free + [t[e] for t, h in zip(table, held) for e in range(pages_of(h, page))]
        assert sorted(owned) == list(range(P))
    assert done > 50


@pytest.mark.parametrize("mask", ["none", "causal", "tree"])
@pytest.mark.parametrize("H,KV", [(4, 4), (6, 2), (3, 1)])
def test_attention_against_torch(mask, H, KV):
    rng = np.random.default_rng(H)
    n, L, D = 7, 19, 16
    q, k, v = rng.standard_normal((n, H, D)), rng.standard_normal((L, KV, D)), rng.standard_normal((L, KV, D))
    bits = [int(rng.integers(0, 1 << n)) | 1 << i for i in range(n)]
    seen = sees(mask, n, L, bits)
    t = lambda x: torch.from_numpy(x).permute(1, 0, 2)[None]
    rep = lambda x: np.repeat(x, H // KV, axis=1)
    ref = F.scaled_dot_product_attention(t(q), t(rep(k)), t(rep(v)), attn_mask=torch.from_numpy(seen))
    o, absum, mag = attend(q, k, v, seen)
    np.testing.assert_allclose(o, ref[0].permute(1, 0, 2).numpy(), rtol=0, atol=1e-13)
    assert np.all(absum >= np.abs(o) - 1e-12) and np.all(mag > 0)


def test_masks_by_hand():
    assert sees("causal", 2, 4).tolist() == [[1, 1, 1, 0], [1, 1, 1, 1]]
    assert sees("tree", 2, 3, [0b01, 0b10]).tolist() == [[1, 1, 0], [1, 0, 1]]
    assert sees("none", 1, 2).all()
    # a call with more rows than keys: the first rows stand before the first key
    assert sees("causal", 3, 2).tolist() == [[0, 0], [1, 0], [1, 1]]


def test_unseen_keys_are_not_computed_with():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((2, 2, 8)), rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8))
    k[2], v[2] = np.nan, np.inf
    seen = np.array([[1, 1, 0], [0, 0, 0]], bool)
    o, _, _ = attend(q, k, v, seen)
    assert np.isfinite(o).all() and not o[1].any()


def test_pages_hold_the_packed_rows():
    rng = np.random.default_rng(6)
    pool_k, pool_v = rng.standard_normal((5, 2, 16, 4)), rng.standard_normal((5, 2, 16, 4))
    k, v, ok = cached_rows(pool_k, pool_v, [3, 0, 9], 35)
    assert ok.tolist() == [True] * 32 + [False] * 3
    assert np.array_equal(k[17], pool_k[0, :, 1]) and np.array_equal(v[5], pool_v[3, :, 5])
