"""Rotary positions of rows, alone and on the way into pages, and the positions of a step's rows, against the float64
oracle.

Error bound of a turned element, u cos t - v sin t times m in fp32: the angle is reduced in fp64 (position * 2^-53 turns,
nothing here) and rounded to fp32 as a part of a turn, at most half a one, so off by 2^-26 turns = 2 pi 2^-26 < 2^-23
radians; sine and cosine are good to 2^-22 of one (their own error and m's product); the products and the sum round three
times.  So m (|u| + |v|) (2^-23 + 2^-22 + 3 * 2^-24) < m (|u| + |v|) 2^-20.8, and the result's own rounding, half a step."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from gqa_util import TYPES, U, desc, torch_types
from oracle.budget import frequencies, rotate

pytestmark = pytest.mark.gpu
KINDS = {"plain": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(gen, *shape):
    import torch
    return torch.empty(shape, device="cuda").normal_(0.0, 1.0, generator=gen)


def _rope(S, layout, rot, scaling="plain", factor=1.0, theta=10000.0, original=2048, magnitude=0.0):
    import torch
    high = 32.0 if scaling == "ramp" else 4.0
    r = S.seer_rope_desc(["half", "pairs"].index(layout), rot, KINDS[scaling], original, theta, factor, 1.0, high, magnitude)
    return r, lambda D: torch.tensor(S.seer_rope_turns(r, D), dtype=torch.float64, device="cuda")


def _freq(rot, scaling="plain", factor=1.0, theta=10000.0, original=2048):
    return frequencies(rot, theta, scaling, factor, 1.0, 32.0 if scaling == "ramp" else 4.0, original)


def _check(got, x, pos, freq, layout, kind, what, inverse=False, m=1.0):
    """got, x [n, heads, D]; rows with a position below zero are not looked at."""
    R = 2 * len(freq)
    live = np.asarray(pos) >= 0
    want = rotate(x, np.maximum(pos, 0), freq, layout, inverse, m)
    assert np.array_equal(got[live][..., R:], x[live][..., R:]), "%s: dims behind the turned ones" % what
    a = np.arange(R // 2) * (2 if layout == "pairs" else 1)
    b = a + (1 if layout == "pairs" else R // 2)
    size = np.zeros(x.shape)
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    tol = m * size * 2.0 ** -20.8 + np.abs(want) * U[kind] * 1.01 + 1e-30
    worst = (np.abs(got - want) / tol)[live][..., :R].max() if live.any() else 0.0
    assert worst <= 1.0, "%s: %.3g of the bound" % (what, worst)
    return worst


SHAPES = [("bf16", 4, 2, 128), ("bf16", 7, 1, 64), ("f32", 3, 3, 80), ("f32", 2, 1, 4), ("f32", 32, 8, 128)]


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("kind,H,KV,D", SHAPES)
def test_parts_of_a_head(S, kind, H, KV, D, layout):
    """Every part of the head that can turn in one of the ways that the kernel takes: whole pieces, odd ends, one pair."""
    t = torch_types(kind)[0]
    for rot in sorted({D, 2, D // 2 // 2 * 2, max(2, D - 16), max(2, D - 6), min(D, 10), min(D, 34)}):
        n, gen = 37, _gen(rot)
        rope, turns = _rope(S, layout, rot)
        q, k = _normal(gen, n, H * D + 32).to(t), _normal(gen, n, KV * D).to(t)
        qo, ko = _normal(gen, n, H * D + 16).to(t), _normal(gen, n, KV * D).to(t)
        q0, qo0, ko0 = host(q), host(qo), host(ko)
        pos = np.arange(n) * 3
        pos[5], pos[36] = -1, -7
        S.seer_rope_rows(desc(S, kind, H, KV, D), rope, turns(D), 0, q, q.stride(0), k, k.stride(0), qo, qo.stride(0), ko,
                         ko.stride(0), n, dev(pos))
        got_q, got_k = host(qo), host(ko)
        assert (got_q[:, H * D:] == qo0[:, H * D:]).all() and (got_q[pos < 0] == qo0[pos < 0]).all()
        assert (got_k[pos < 0] == ko0[pos < 0]).all() and (host(q) == q0).all()
        w = _check(got_q[:, :H * D].reshape(n, H, D), q0[:, :H * D].reshape(n, H, D), pos, _freq(rot), layout, kind, "q")
        w = max(w, _check(got_k.reshape(n, KV, D), host(k).reshape(n, KV, D), pos, _freq(rot), layout, kind, "k"))
        log("  %s %s dim %d rot %d: %.3g of the bound" % (kind, layout, D, rot, w))


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("scaling", list(KINDS))
def test_scaling_and_far_positions(S, scaling, layout):
    """Positions up to 2^31 - 1: an angle in fp32 would be off by hundreds of turns."""
    H, KV, D, n = 2, 1, 128, 40
    pos = np.concatenate([np.arange(20), 10 ** np.arange(10), [2 ** 31 - 1] * 2, 2 ** 24 + np.arange(8)])
    rope, turns = _rope(S, layout, D, scaling, 8.0, 500000.0)
    q, k = _normal(_gen(1), n, H * D), _normal(_gen(2), n, KV * D)
    x = host(q).reshape(n, H, D)
    S.seer_rope_rows(desc(S, "f32", H, KV, D), rope, turns(D), 0, q, H * D, k, KV * D, q, H * D, k, KV * D, n, dev(pos))
    # the oracle's own angle: position * 2^-53 * 2 pi * f / f, at most 2^31 * 2^-53 * 7 radians, far below the bound
    m = 0.1 * np.log(8.0) + 1.0 if scaling == "ramp" else 1.0
    _check(host(q).reshape(n, H, D), x, pos, _freq(D, scaling, 8.0, 500000.0), layout, "f32", scaling, m=m)


@pytest.mark.parametrize("kind,H,KV,D", SHAPES[:3])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_in_place_and_back(S, kind, H, KV, D, layout):
    """Rows of one projection, q | k | v, turned in place: as out of place, bit for bit; the inverse is the gradient."""
    import torch
    t, n = torch_types(kind)[0], 130
    for rot in (D, 10):
        rope, turns = _rope(S, layout, rot, magnitude=1.25)
        d, tt, pos = desc(S, kind, H, KV, D), turns(D), dev(np.arange(n) - 2)
        qkv = _normal(_gen(3), n, (H + 2 * KV) * D).to(t)
        before = qkv.clone()
        q, k = qkv[:, :H * D], qkv[:, H * D:(H + KV) * D]
        s = qkv.stride(0)
        qo, ko = q.clone().contiguous(), k.clone().contiguous()
        S.seer_rope_rows(d, rope, tt, 0, q, s, k, s, qo, H * D, ko, KV * D, n, pos)
        assert torch.equal(qkv, before)
        S.seer_rope_rows(d, rope, tt, 0, q, s, k, s, q, s, k, s, n, pos)
        assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, (H + KV) * D:], before[:, (H + KV) * D:])
        only = before.clone()
        S.seer_rope_rows(d, rope, tt, 0, None, 0, only[:, H * D:], s, None, 0, only[:, H * D:], s, n, pos)
        assert torch.equal(only[:, :H * D], before[:, :H * D]) and torch.equal(only[:, H * D:(H + KV) * D], k)
        back = ko.clone()
        S.seer_rope_rows(d, rope, tt, S.SEER_ROPE_INVERSE, None, 0, ko, KV * D, None, 0, back, KV * D, n, pos)
        _check(host(back).reshape(n, KV, D), host(ko).reshape(n, KV, D), np.arange(n) - 2, _freq(rot), layout, kind, "back",
               inverse=True, m=1.25)


def test_gradient(S):
    """The inverse takes a gradient back: against differences of sum(g * rotated), which is linear in the row."""
    H, KV, D, n = 1, 1, 8, 3
    rope, turns = _rope(S, "pairs", 6, magnitude=1.5)
    d, tt, pos = desc(S, "f32", H, KV, D), turns(D), dev(np.array([1, 5, 1000]))
    x, g = _normal(_gen(4), n, D), _normal(_gen(5), n, D)

    def turn(a, flags):
        out = a.clone()
        S.seer_rope_rows(d, rope, tt, flags, out, D, None, 0, out, D, None, 0, n, pos)
        return host(out)

    got = turn(g, S.SEER_ROPE_INVERSE)
    want = np.zeros((n, D))
    for j in range(D):
        step = x.clone()
        step[:, j] += 1.0                            # a whole step: the function is linear
        want[:, j] = (host(g) * (turn(step, 0) - turn(x, 0))).sum(1)
    # 16 products of values up to 5, each off by 2^-20 of them
    assert np.abs(got - want).max() <= 16 * 5 * 5 * 2.0 ** -20


def test_as_the_layer_turns(S):
    """The layer's own rotary embedding (half layout, whole heads) to the oracle, beside this one's."""
    H, KV, D, n = 4, 4, 128, 50
    rope, turns = _rope(S, "half", D, theta=500000.0)
    q, k = _normal(_gen(6), n, H * D), _normal(_gen(7), n, KV * D)
    from oracle.rope import apply_rope
    want = apply_rope(host(q), np.arange(n), H, 500000.0)
    S.seer_rope_rows(desc(S, "f32", H, KV, D), rope, turns(D), 0, q, H * D, k, KV * D, q, H * D, k, KV * D, n,
                     dev(np.arange(n)))
    assert np.abs(host(q) - want).max() <= 2 * 6 * 2.0 ** -20.8        # |u| + |v| below 12


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("kind,H,KV,D,page,rot", [("bf16", 4, 2, 128, 16, 128), ("v16", 7, 1, 64, 64, 32),
                                                  ("f32", 3, 3, 80, 32, 10), ("bf16", 32, 8, 128, 256, 112)])
def test_store(S, kind, H, KV, D, page, rot, layout):
    import torch
    qt, vt = torch_types(kind)
    n, P = 77, 9
    gen = _gen(8)
    rope, turns = _rope(S, layout, rot)
    buf = _normal(gen, n, (H + 2 * KV) * D).to(qt)
    q, k = buf[:, :H * D], buf[:, H * D:(H + KV) * D]
    v = buf.view(vt)[:, (H + KV) * D:]
    v.copy_(_normal(gen, n, KV * D))
    qo = torch.full((n, H * D), 9.0, dtype=qt, device="cuda")
    pool = torch.full((P, 2, KV, page, D), 3.0, dtype=qt, device="cuda")
    pool.view(vt)[:, 1] = 3.0
    weight = torch.full((P, KV, page), 5.0, device="cuda")
    number = torch.full((P, KV, page), -5, dtype=torch.int32, device="cuda")
    slots = np.random.default_rng(1).permutation(P * page)[:n]
    pos = np.arange(n) * 2 + 1
    slots[3], slots[10], pos[20] = -1, P * page + 4, -1
    live = (slots >= 0) & (slots < P * page) & (pos >= 0)
    S.seer_kv_store_rope(desc(S, kind, H, KV, D), S.seer_page_desc(page, P, 4), rope, turns(D), q, q.stride(0), qo, H * D, k,
                         k.stride(0), v, v.stride(0), n, dev(pos), dev(slots), pool, weight, number)
    got_q, got_k = host(qo).reshape(n, H, D), host(pool)[:, 0]
    got_v = host(pool.view(vt)[:, 1])
    assert (got_q[~live] == 9.0).all()
    at = np.where(live, pos, -1)
    _check(got_q, host(q).reshape(n, H, D), at, _freq(rot), layout, TYPES[kind][0], "q")
    pages, offs = slots[live] // page, slots[live] % page
    _check(got_k[pages, :, offs], host(k).reshape(n, KV, D)[live], pos[live], _freq(rot), layout, TYPES[kind][0], "k")
    assert np.array_equal(got_v[pages, :, offs], host(v).reshape(n, KV, D)[live])
    rest = np.ones((P, page), bool)
    rest[pages, offs] = False
    assert (got_k.transpose(0, 2, 1, 3)[rest] == 3.0).all() and (got_v.transpose(0, 2, 1, 3)[rest] == 3.0).all()
    w, m = host(weight).transpose(0, 2, 1), host(number).transpose(0, 2, 1)
    assert (w[rest] == 5.0).all() and (m[rest] == -5).all()
    assert (w[pages, offs] == 0.0).all() and (m[pages, offs] == pos[live][:, None]).all()
    # without queries and marks: the same keys
    again = torch.full_like(pool, 3.0)
    again.view(vt)[:, 1] = 3.0
    S.seer_kv_store_rope(desc(S, kind, H, KV, D), S.seer_page_desc(page, P, 4), rope, turns(D), None, 0, None, 0, k,
                         k.stride(0), v, v.stride(0), n, dev(pos), dev(slots), again, None, None)
    assert torch.equal(again.view(torch.int16 if qt is not torch.float32 else torch.int32),
                       pool.view(torch.int16 if qt is not torch.float32 else torch.int32))


def test_many_rows(S):
    """More rows than a launch has waves at once, the last ones padding."""
    import torch
    H, KV, D, n = 2, 1, 64, 40000
    rope, turns = _rope(S, "half", D)
    q = _normal(_gen(9), n, H * D).to(torch.bfloat16)
    k = _normal(_gen(10), n, KV * D).to(torch.bfloat16)
    x, pos = host(q), np.arange(n)
    pos[39000:] = -1
    S.seer_rope_rows(desc(S, "bf16", H, KV, D), rope, turns(D), 0, q, H * D, k, KV * D, q, H * D, k, KV * D, n, dev(pos))
    got = host(q)
    assert np.array_equal(got[39000:], x[39000:])
    at = np.array([0, 1, 3, 4, 12345, 38999])
    _check(got[at].reshape(-1, H, D), x[at].reshape(-1, H, D), pos[at], _freq(D), "half", "bf16", "rows")


@pytest.mark.parametrize("B", [1, 3, 300])
def test_row_positions(S, B):
    import torch
    r = np.random.default_rng(B)
    lens = r.integers(0, 9, B)
    cu = np.concatenate([[0], np.cumsum(lens)])
    used, seen, base = r.integers(-1, 10, B), r.integers(0, 1000, B), r.integers(0, 1000, B)
    rows = int(cu[-1]) + 70
    real = np.minimum(np.maximum(used, 0), lens)

    def want(start, real):
        out = np.full(rows, -1)
        for b in range(B):
            out[cu[b]:cu[b] + real[b]] = start[b] + np.arange(real[b])
        return out

    for s, ba, u in ((seen, None, None), (seen, base, used), (None, None, used), (None, base, None)):
        pos, nxt = dev(np.full(rows, 77)), dev(np.full(B, 77))
        status = dev(np.array([0]))
        n = lens if u is None else real
        start = ba if ba is not None else (s if s is not None else np.zeros(B, int))
        opt = lambda x: None if x is None else dev(x)
        S.seer_row_positions(dev(cu), opt(u), B, opt(s), opt(ba), status, rows, pos, nxt)
        assert np.array_equal(host(pos), want(start, n)) and np.array_equal(host(nxt), start + n)
        status.fill_(4)                              # a refused plan: nothing has moved on
        S.seer_row_positions(dev(cu), opt(u), B, opt(s), opt(ba), status, rows, pos, nxt)
        assert (host(pos) == -1).all() and np.array_equal(host(nxt), np.zeros(B) if s is None else s)
        S.seer_row_positions(dev(cu), opt(u), B, opt(s), opt(ba), None, 0, None, nxt)
        assert np.array_equal(host(nxt), start + n)
