"""The attention weight of cached tokens against the float64 oracle: types, head layouts, lengths around the tiles,
masks that leave rows empty, unseen NaN, pages that are none, rows that do not count, long caches, streams, recordings.

Error bound of a weight, a sum of probabilities: a score is a sum of D products in fp32, off by at most D 2^-23 times
m = scale sum |q k| whatever the order, and meets roundings of size 2^-24 m (the product with log2 e, the differences
with the maximum and with the row's logarithm, at most 2 m each): d = (D 2^-23 + 16 * 2^-24) m + 2^-21, the last the
exponential's.  The row's sum is off by d and by n 2^-24 for its n terms, its logarithm (up to 31) by 2^-20; so each p by
2 d + (n + 16) 2^-24 + 2^-20, and the sum over them and the old weight by its own length times 2^-24."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from gqa_util import desc, torch_types, words_of
from oracle.budget import weights
from oracle.paged import cached_rows, sees

pytestmark = pytest.mark.gpu


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


class Call:
    """Requests with past[b] cached tokens before lens[b] rows, of which used[b] are real."""

    def __init__(self, S, kind, H, KV, D, past, lens, used=None, page=16, pad=5, factor=1.0, seed=1, scale=0.0, bits=None,
                 width=None, batch=None):
        import torch
        self.S, self.kind, self.shape, self.page, self.scale = S, kind, (H, KV, D), page, scale or None
        self.past, self.lens = past, lens
        self.used = list(lens) if used is None else [max(0, min(u, n)) for u, n in zip(used, lens)]
        self.B, self.bits = len(lens), bits
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(int)
        self.rows = max(int(self.cu[-1]) + pad, 1)
        gen, qt = _gen(seed), torch_types(kind)[0]
        self.kv_len = [p + u for p, u in zip(past, self.used)]
        need = [-(-max(n, 0) // page) for n in self.kv_len]
        self.W = width or max(max(need), 1)
        self.P = sum(need) + 3
        ids = np.random.default_rng(seed).permutation(self.P)
        table, at = np.full((self.B, self.W), -1), 0
        for b, n in enumerate(need):
            table[b, :n] = ids[at:at + n]
            at += n
        self.table = table
        self.q = _normal(gen, self.rows, H * D + 16).mul_(factor).to(qt)[:, :H * D]
        self.pool = _normal(gen, self.P, 2, KV, page, D).to(qt)
        self.pool[:, 1] = float("nan")               # V is not looked at
        self.prev = _normal(gen, self.P, KV, page).abs_()
        self.desc, self.pages = desc(S, kind, H, KV, D, scale), S.seer_page_desc(page, self.P, self.W)
        self.bits_d = None
        if bits is not None:
            words = max(1, -(-max(lens) // 64))
            self.bits_d = torch.zeros(self.rows, words, dtype=torch.int64, device="cuda")
            self.bits_d[:len(bits)] = torch.from_numpy(words_of(bits, words)).cuda()
        self.cu_d, self.kv_d = dev(self.cu), dev(np.array(self.kv_len))
        self.used_d = None if used is None else dev(np.array(used))
        n = S.seer_attn_weights_workspace_bytes(self.desc, self.pages, self.rows, self.B)
        self.ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
        self.weight = torch.full((self.P, KV, page), 7.0, device="cuda")
        self.table_d = dev(table)

    def run(self, mask, last=0, decay=1.0, prev=True, weight=None, stream=None, ws=None):
        m = dict(none=0, causal=1, tree=2)[mask]
        self.S.seer_attn_weights(self.desc, self.pages, m, self.q, self.q.stride(0), self.rows, self.cu_d, self.used_d, self.B,
                                 last, self.pool, self.table_d, self.kv_d, self.bits_d,
                                 0 if self.bits_d is None else self.bits_d.shape[1], decay, self.prev if prev else None,
                                 self.weight if weight is None else weight, self.ws if ws is None else ws, stream=stream)

    def check(self, mask, last=0, decay=1.0, prev=True, got=None, requests=None):
        H, KV, D = self.shape
        got = host(self.weight) if got is None else got
        q, pool_k, old = host(self.q).reshape(-1, H, D), host(self.pool[:, 0]), host(self.prev)
        written, worst = np.zeros(got.shape, bool), 0.0
        for b in range(self.B):
            u, L, s = self.used[b], self.kv_len[b], self.cu[b]
            if u == 0:
                continue
            c = min(u, last) if last else u
            k, _, ok = cached_rows(pool_k, pool_k, self.table[b], L)
            for j in range(L):
                if ok[j]:
                    written[self.table[b][j // self.page], :, j % self.page] = True
            if requests is not None and b not in requests:
                continue
            seen = sees(mask, u, L, None if self.bits is None else self.bits[s:s + u])[u - c:] & ok[None, :]
            w, mag, keys = weights(q[s + u - c:s + u], k, seen, self.scale)
            before = np.zeros((L, KV))
            for j in range(L):
                if prev and decay and ok[j]:
                    before[j] = old[self.table[b][j // self.page], :, j % self.page]
            want = decay * before + w
            tol = (2 * (D * 2.0 ** -23 + 16 * 2.0 ** -24) * mag + (keys + 16 * w) * 2.0 ** -24 + 3 * 2.0 ** -20 * w
                   + (c * (H // KV) + 4) * 2.0 ** -24 * want) * 1.01 + 2.0 ** -60
            for j in range(L):
                if not ok[j]:
                    continue
                g = got[self.table[b][j // self.page], :, j % self.page]
                e = np.abs(g - want[j]) / tol[j]
                assert (e <= 1.0).all(), "request %d token %d: %r for %r (%.3g of the bound)" % (b, j, g, want[j], e.max())
                worst = max(worst, float(e.max()))
        assert (got[~written] == 7.0).all(), "written outside the requests' tokens"
        return worst


SHAPES = [("bf16", 4, 4, 128), ("bf16", 8, 2, 128), ("bf16", 7, 1, 64), ("v16", 6, 2, 64), ("f32", 4, 2, 64),
          ("f32", 3, 1, 80), ("f32", 5, 5, 4), ("bf16", 16, 1, 128)]
PAST = [0, 1, 15, 31, 32, 63, 64, 65, 127, 130, 200, 0]
LENS = [1, 1, 1, 1, 3, 0, 1, 2, 33, 5, 17, 70]


def _bits(lens, seed=0):
    r, out = np.random.default_rng(seed), []
    for n in lens:
        seen = []
        for i in range(n):
            up = int(r.integers(-1, i)) if i else -1
            seen.append((seen[up] if up >= 0 else 0) | 1 << i)
        out += seen
    return out


@pytest.mark.parametrize("mask", ["causal", "none", "tree"])
@pytest.mark.parametrize("kind,H,KV,D", SHAPES)
def test_lengths(S, kind, H, KV, D, mask):
    log("%s %s heads %d/%d dim %d" % (mask, kind, H, KV, D))
    c = Call(S, kind, H, KV, D, PAST, LENS, bits=_bits(LENS) if mask == "tree" else None)
    c.run(mask, decay=0.5)
    log("  %.3g of the bound" % c.check(mask, decay=0.5))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_single_tokens(S, kind):
    for H, KV, D in ((32, 8, 128), (14, 2, 64), (8, 8, 64)):
        c = Call(S, kind, H, KV, D, [0, 793, 5, 64, 300], [1] * 5, pad=0, page=64)
        c.run("causal", prev=False)
        c.check("causal", prev=False)


@pytest.mark.parametrize("last", [1, 4, 32, 64])
def test_last_rows(S, last):
    used = [0, 1, 1, 1, 2, 0, 1, 2, 20, 5, 17, 70]
    for kind in ("bf16", "f32"):
        for mask in ("causal", "none", "tree"):
            c = Call(S, kind, 4, 2, 64, PAST, LENS, used=used, bits=_bits(LENS) if mask == "tree" else None)
            c.run(mask, last=last)
            c.check(mask, last=last)


def test_old_weights(S):
    """In place, apart, none, and none that are read with decay 0 (they are NaN here)."""
    import torch
    c = Call(S, "bf16", 4, 2, 128, [40, 3], [5, 20])
    c.run("causal", decay=0.9)
    apart = c.weight.clone()
    c.check("causal", decay=0.9)
    place = c.prev.clone()
    c.S.seer_attn_weights(c.desc, c.pages, 1, c.q, c.q.stride(0), c.rows, c.cu_d, None, c.B, 0, c.pool, c.table_d, c.kv_d, None,
                          0, 0.9, place, place, c.ws)
    live = apart != 7.0
    assert torch.equal(place[live], apart[live]) and torch.equal(place[~live], c.prev[~live])
    c.run("causal", prev=False)
    none = c.weight.clone()
    c.prev.fill_(float("nan"))
    c.weight.fill_(7.0)
    c.run("causal", decay=0.0)
    assert torch.equal(none, c.weight)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_rows_that_see_nothing(S, kind):
    """Empty bits; a cache that is shorter than the call says, so that its first rows stand before the first key."""
    bits = [0, 1, 0, 4, 8, 0, 0, 2]
    c = Call(S, kind, 4, 2, 64, [0, 0], [5, 3], bits=bits)
    c.run("tree")
    c.check("tree")
    c = Call(S, kind, 4, 2, 64, [-3, 4], [8, 2])
    c.kv_len = [5, 6]
    c.run("causal")
    c.check("causal")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_unseen_nan(S, kind):
    """Keys past a row's position, past the end and on pages that are none reach no weight; a row's padding neither."""
    import torch
    c = Call(S, kind, 4, 2, 64, [70, 20, 33], [40, 6, 1], used=[30, 6, 1])
    c.run("causal")
    clean = c.weight.clone()
    c.q[30:40] = float("nan")
    c.q[int(c.cu[-1]):] = float("nan")
    flat = c.pool[:, 0]
    for b in range(3):
        for j in range(c.kv_len[b], c.W * 16):
            if c.table[b, j // 16] >= 0:
                flat[c.table[b, j // 16], :, j % 16] = float("nan")
    used = {int(x) for x in c.table.reshape(-1)}
    for p in range(c.P):
        if p not in used:
            c.pool[p] = float("nan")
    c.weight.fill_(7.0)
    c.run("causal")
    assert torch.equal(clean, c.weight)
    # the last row's own key: only the last row sees it, and all that it sees is NaN then
    page, slot = c.table[0, 99 // 16], 99 % 16
    c.pool[page, 0, :, slot] = float("nan")
    c.run("none", last=1)                          # everything of request 0
    assert torch.isnan(c.weight[page, :, slot]).all()
    # causal, of the rows before: weights of the first 99 keys come from rows 0..28 and the last one, which is NaN
    c.used_d = dev(np.array([29, 6, 1]))
    c.kv_d = dev(np.array([99, 26, 34]))
    c.weight.fill_(7.0)
    c.run("causal")
    first = [int(c.table[0, j // 16]) for j in range(99)]
    assert torch.isfinite(c.weight[first[0]]).all() and not torch.isnan(c.weight).any()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_pages_that_are_none(S, kind):
    """Their tokens are seen by no row, and nothing is written for them."""
    c = Call(S, kind, 4, 2, 64, [120, 70], [9, 1])
    c.table[0, 2], c.table[0, 5], c.table[1, 0] = -1, c.P, 1 << 30
    c.table_d = dev(c.table)
    for mask in ("causal", "none"):
        c.weight.fill_(7.0)
        c.run(mask)
        c.check(mask)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_page_sizes(S, kind, page):
    c = Call(S, kind, 4, 2, 64, [500, 255, 256, 1], [3, 1, 40, 2], page=page, width=40)
    c.run("causal")
    c.check("causal")


@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 64)])
def test_long(S, kind, H, KV, D):
    """Many parts of many tiles, beside a short request."""
    c = Call(S, kind, H, KV, D, [5000, 7], [1, 1], page=64)
    c.run("causal")
    c.check("causal")
    c = Call(S, kind, H, KV, D, [1500, 0, 64], [200, 3, 130], page=64)
    for mask in ("causal", "none"):
        c.run(mask, last=20)
        c.check(mask, last=20)
        c.run(mask)
        c.check(mask, requests=[1, 2])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_scores_that_rise(S, kind):
    """Large scores whose maximum comes late."""
    c = Call(S, kind, 2, 1, 64, [700, 100], [2, 200], factor=6.0)
    ramp = dev(np.linspace(0.2, 3.0, c.P), "f32")[:, None, None, None]
    c.pool[:, 0] = (c.pool[:, 0].float().abs() * ramp).to(c.pool.dtype)
    c.q.copy_(c.q.float().abs())
    c.run("causal")
    c.check("causal")


def test_scale(S):
    c = Call(S, "bf16", 4, 2, 64, [70, 0], [3, 10], scale=0.3)
    c.run("causal")
    c.check("causal")


def test_many_requests(S):
    """More requests than threads, most without rows."""
    r = np.random.default_rng(3)
    lens = [int(x) for x in r.integers(0, 3, 700)]
    past = [int(x) for x in r.integers(0, 40, 700)]
    for kind in ("bf16", "f32"):
        c = Call(S, kind, 4, 2, 64, past, lens)
        c.run("causal")
        c.check("causal", requests=set(range(0, 700, 37)))


def test_bits_are_the_same_each_time(S):
    import torch
    c = Call(S, "bf16", 8, 2, 128, [3000, 100, 40], [7, 100, 1], page=64)
    c.run("causal")
    first = c.weight.clone()
    for _ in range(3):
        c.weight.fill_(7.0)
        c.run("causal")
        assert torch.equal(first, c.weight)


def test_streams_and_recordings(S):
    """Two streams with workspaces of their own at once; a recording replayed with other inputs and its own eager
    call between."""
    import torch
    from paper_2607_14557_amd.runner import record
    a, b = Call(S, "bf16", 8, 2, 128, [900, 30], [3, 50], seed=1), Call(S, "bf16", 8, 2, 128, [400, 64], [1, 90], seed=2)
    want = []
    for c in (a, b):
        c.run("causal")
        want.append(c.weight.clone())
        c.weight.fill_(7.0)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.run("causal", stream=s1)
        b.run("causal", stream=s2)
    torch.cuda.synchronize()
    assert torch.equal(a.weight, want[0]) and torch.equal(b.weight, want[1])
    graph = record(lambda: a.run("causal", stream=s1), s1)
    for i in range(4):
        a.q.copy_(_normal(_gen(20 + i), *a.q.shape))
        a.weight.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay(s1)
        torch.cuda.synchronize()
        got = a.weight.clone()
        a.weight.fill_(7.0)
        a.run("causal")
        torch.cuda.synchronize()
        assert torch.equal(got, a.weight), "replay %d" % i
