"""Attention with grouped heads over packed prompts and over pages, against the
float64 oracle: types, head layouts, lengths around the tiles, padding, masks
that leave rows empty, NaN and infinities where a row does not look, pages that
end inside a tile or are none, long contexts, strides, streams, recordings."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from gqa_util import TYPES, check, desc, torch_types, words_of, workspace
from oracle.paged import cached_rows, sees

pytestmark = pytest.mark.gpu
LENS = [1, 2, 31, 32, 33, 0, 63, 64, 65, 127, 129, 200]


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


def _normal(gen, *shape):
    import torch
    return torch.empty(shape, device="cuda").normal_(0.0, 1.0, generator=gen)


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class Prompt:
    """Packed q | k | v rows with a gap behind them, and the call on them."""

    def __init__(self, S, kind, H, KV, D, lens, used=None, pad=5, factor=1.0, seed=1, scale=0.0):
        import torch
        self.S, self.kind, self.shape = S, kind, (H, KV, D)
        self.qt, self.vt = torch_types(kind)
        self.lens, self.used = lens, used
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(int)
        self.T, gen = int(self.cu[-1]), _gen(seed)
        self.rows = max(self.T + pad, 1)
        gap = 16
        buf = _normal(gen, self.rows, (H + 2 * KV) * D + gap).to(self.qt)
        self.q, self.k = buf[:, :H * D], buf[:, H * D:(H + KV) * D]
        self.q.mul_(factor)
        self.v = buf.view(self.vt)[:, (H + KV) * D:(H + 2 * KV) * D]
        self.v.copy_(_normal(gen, self.rows, KV * D))
        self.out = torch.full((self.rows, H * D + 32), 9.0, dtype=self.qt, device="cuda")
        self.desc = desc(S, kind, H, KV, D, scale)
        self.scale = scale or None
        self.cu_d, self.used_d = dev(self.cu), None if used is None else dev(np.asarray(used))
        self.ws = workspace(S, self.desc, self.rows, len(lens))

    def run(self, mask, stream=None, out=None):
        out = self.out if out is None else out
        self.S.seer_attn_prompt(self.desc, mask, self.q, self.q.stride(0), self.k, self.k.stride(0), self.v,
                                self.v.stride(0), out, out.stride(0), self.rows, self.cu_d, self.used_d, len(self.lens),
                                self.ws, stream=stream)

    def check(self, mask, rows=None):
        H, KV, D = self.shape
        T, worst = self.T, 0.0
        got = host(self.out)
        assert (got[T:] == 9.0).all() and (got[:, H * D:] == 9.0).all(), "written outside the rows"
        q, k, v = host(self.q).reshape(-1, H, D), host(self.k).reshape(-1, KV, D), host(self.v).reshape(-1, KV, D)
        got = got[:, :H * D].reshape(-1, H, D)
        for b, (s, n) in enumerate(zip(self.cu, self.lens)):
            u = n if self.used is None else max(0, min(self.used[b], n))
            assert not got[s + u:s + n].any(), "padding rows get zeros"
            at = None if rows is None else [r for r in rows if r < u]
            if u and (at is None or at):
                worst = max(worst, check(got[s:s + u], q[s:s + u], k[s:s + u], v[s:s + u], sees(mask, u, u),
                                         *TYPES[self.kind], "sequence %d" % b, rows=at, scale=self.scale))
        return worst


SHAPES = [("bf16", 4, 4, 128), ("bf16", 8, 2, 128), ("bf16", 7, 1, 64), ("bf16", 6, 2, 64), ("v16", 4, 2, 128),
          ("v16", 3, 3, 64), ("f32", 4, 2, 64), ("f32", 3, 1, 80), ("f32", 2, 2, 128), ("f32", 5, 5, 4)]


@pytest.mark.parametrize("mask", ["causal", "none"])
@pytest.mark.parametrize("kind,H,KV,D", SHAPES)
def test_prompt_lengths(S, kind, H, KV, D, mask):
    log("prompt %s %s heads %d/%d dim %d" % (mask, kind, H, KV, D))
    p = Prompt(S, kind, H, KV, D, LENS)
    p.run(S.SEER_MASK_CAUSAL if mask == "causal" else S.SEER_MASK_NONE)
    log("  %.3g of the bound" % p.check(mask))


@pytest.mark.parametrize("kind,H,KV,D", SHAPES[1:8:2])
def test_prompt_padding(S, kind, H, KV, D):
    log("padded prompt %s heads %d/%d dim %d" % (kind, H, KV, D))
    used = [0, 1, 30, 40, -3, 0, 1, 64, 64, 5, 129, 128]
    for mask, m in (("causal", S.SEER_MASK_CAUSAL), ("none", S.SEER_MASK_NONE)):
        p = Prompt(S, kind, H, KV, D, LENS, used=used)
        p.run(m)
        p.check(mask)


@pytest.mark.parametrize("kind", list(TYPES))
def test_prompt_one_row(S, kind):
    for H, KV, D in ((1, 1, 128), (32, 8, 128), (14, 2, 64)):
        p = Prompt(S, kind, H, KV, D, [1], pad=0)
        p.run(S.SEER_MASK_CAUSAL)
        p.check("causal")


@pytest.mark.parametrize("kind", list(TYPES))
def test_prompt_scores_that_rise(S, kind):
    """Large scores whose maximum comes late: the reference maximum moves, and moves more than fp16 holds."""
    p = Prompt(S, kind, 2, 1, 128, [300, 700], factor=6.0)
    ramp = dev(np.linspace(0.2, 3.0, p.rows), "f32")[:, None]
    p.k.copy_(p.k.float().abs() * ramp)
    p.q.copy_(p.q.float().abs())
    p.run(S.SEER_MASK_CAUSAL)
    p.check("causal", rows=[0, 1, 63, 64, 100, 255, 256, 299, 500, 699])


def test_prompt_scale(S):
    p = Prompt(S, "bf16", 4, 2, 64, [70, 10], scale=0.3)
    p.run(S.SEER_MASK_CAUSAL)
    p.check("causal")


@pytest.mark.parametrize("kind", list(TYPES))
def test_prompt_long(S, kind):
    """Long rows of tiles, several to a sequence, sampled rows."""
    n = 3001 if kind != "f32" else 1501
    p = Prompt(S, kind, 4, 2, 128, [n, 5, 777])
    p.run(S.SEER_MASK_CAUSAL)
    p.check("causal", rows=[0, 1, 127, 128, 500, 776, 1023, 1500, 2047, 3000])


@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 4, 2, 128), ("bf16", 2, 1, 64), ("v16", 2, 2, 128), ("f32", 2, 1, 64)])
def test_prompt_unseen_nan_and_infinity(S, kind, H, KV, D):
    """Values past a row's own position reach it in no way; those that it sees do."""
    p = Prompt(S, kind, H, KV, D, [100, 140], seed=4)
    inf, nan = float("inf"), float("nan")
    p.v[40, 3], p.v[41, 5], p.v[90, 0], p.v[91, 0] = inf, -inf, inf, -inf
    p.v[100 + 130, 2] = nan
    p.v[100 + 77, 1] = -inf
    p.run(S.SEER_MASK_CAUSAL)
    p.check("causal")


def test_prompt_nan_key_is_seen_from_its_own_row_on(S):
    for kind in TYPES:
        p = Prompt(S, kind, 2, 1, 64, [130], seed=5)
        p.k[70, 0] = float("nan")
        p.run(S.SEER_MASK_CAUSAL)
        got = host(p.out)[:130, :128]
        assert np.isfinite(got[:70]).all() and np.isnan(got[70:]).all(), kind


class Paged:
    """Requests in pages of a pool that holds NaN wherever no token lies."""

    def __init__(self, S, kind, H, KV, D, past, new, page=16, used=None, words=0, bits=None, spare=3, seed=1, pad=4,
                 factor=1.0, width=None, first_page=0, kv_len=None):
        import torch
        self.S, self.kind, self.shape, self.page = S, kind, (H, KV, D), page
        self.qt, self.vt = torch_types(kind)
        gen, rng = _gen(seed), np.random.default_rng(seed)
        self.new, self.used = new, list(new) if used is None else used
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(int)
        self.T = int(self.cu[-1])
        self.rows = max(self.T + pad, 1)
        real = [max(0, min(u, n)) for u, n in zip(self.used, new)]
        self.real = real
        self.kv = [p + u for p, u in zip(past, real)]
        need = [-(-n // page) for n in self.kv]
        self.P = sum(need) + spare + first_page
        self.W = width or max(max(need), 1)
        ids = rng.permutation(self.P - first_page) + first_page
        self.table = np.full((len(new), self.W), -1)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.pages = S.seer_page_desc(page, self.P, self.W)
        self.desc = desc(S, kind, H, KV, D)
        if first_page:      # a large pool: only the pages in use are filled
            self.pool = torch.empty(self.P, 2, KV, page, D, dtype=self.qt, device="cuda")
            self.pool[first_page:] = float("nan")
        else:
            self.pool = torch.full((self.P, 2, KV, page, D), float("nan"), dtype=self.qt, device="cuda")
        self.pool.view(self.vt)[first_page:, 1] = float("nan")
        n = max(sum(self.kv), 1)
        k, v = _normal(gen, n, KV * D).to(self.qt), _normal(gen, n, KV * D).to(self.vt)
        self.slots = np.concatenate([[self.table[b, t // page] * page + t % page for t in range(m)]
                                     for b, m in enumerate(self.kv)] + [[]]).astype(int)
        if self.slots.size:
            S.seer_kv_store(self.desc, self.pages, k, KV * D, v, KV * D, self.slots.size, dev(self.slots), self.pool)
        self.q = (_normal(gen, self.rows, H * D) * factor).to(self.qt)
        self.out = torch.full((self.rows, H * D), 9.0, dtype=self.qt, device="cuda")
        self.bits = bits
        self.words = words
        self.bits_d = None if bits is None else torch.zeros(self.rows, words, dtype=torch.int64, device="cuda")
        if bits is not None and self.T:
            self.bits_d[:self.T] = torch.from_numpy(words_of(bits, words)).cuda()
        self.cu_d, self.table_d = dev(self.cu), dev(self.table)
        self.used_d = None if used is None else dev(np.asarray(used))
        self.kv_call = self.kv if kv_len is None else kv_len
        self.kv_d = dev(np.asarray(self.kv_call))
        self.ws = workspace(S, self.desc, self.rows, len(new))

    def run(self, mask, stream=None, out=None, ws=None):
        m = dict(none=self.S.SEER_MASK_NONE, causal=self.S.SEER_MASK_CAUSAL, tree=self.S.SEER_MASK_TREE)[mask]
        out = self.out if out is None else out
        self.S.seer_attn_paged(self.desc, self.pages, m, self.q, self.q.stride(0), out, out.stride(0), self.rows,
                               self.cu_d, self.used_d, len(self.new), self.pool, self.table_d, self.kv_d, self.bits_d,
                               self.words, self.ws if ws is None else ws, stream=stream)

    def check(self, mask, rows=None):
        H, KV, D = self.shape
        got = host(self.out)
        assert (got[self.T:] == 9.0).all(), "rows behind the last sequence are left as they were"
        got, q = got.reshape(-1, H, D), host(self.q).reshape(-1, H, D)
        used_pages = np.unique(self.table[(self.table >= 0) & (self.table < self.P)])
        local = np.full(self.P, -1)
        local[used_pages] = np.arange(used_pages.size)
        if used_pages.size == 0:
            used_pages = np.array([0])
        import torch
        idx = torch.from_numpy(used_pages).cuda()
        pk, pv = host(self.pool[idx, 0]), host(self.pool.view(self.vt)[idx, 1])
        worst = 0.0
        for b, (s, n) in enumerate(zip(self.cu, self.new)):
            u, L = self.real[b], max(0, min(self.kv_call[b], self.W * self.page))
            assert not got[s + u:s + n].any(), "padding rows get zeros"
            if u == 0:
                continue
            row = [local[t] if 0 <= t < self.P else -1 for t in self.table[b]]
            k, v, ok = cached_rows(pk, pv, row, L)
            seen = sees(mask, u, L, None if self.bits is None else
                        [m & ((1 << 64 * self.words) - 1) for m in self.bits[s:s + u]]) & ok[None]
            at = None if rows is None else [r for r in rows if r < u]
            worst = max(worst, check(got[s:s + u], q[s:s + u], k, v, seen, *TYPES[self.kind], "request %d" % b, rows=at))
        return worst


def _tree(rng, n, empty=()):
    bits = []
    for i in range(n):
        up = int(rng.integers(max(-1, i - 6), i)) if i else -1
        bits.append((bits[up] if up >= 0 else 0) | 1 << i)
    for i in empty:
        bits[i] = 0
    return bits


PAST = [0, 1, 15, 16, 17, 47, 48, 63, 64, 65, 127, 128, 129, 300, 0]
NEW = [3, 1, 1, 2, 33, 1, 5, 1, 17, 40, 1, 64, 1, 2, 0]


@pytest.mark.parametrize("mask", ["none", "causal", "tree"])
@pytest.mark.parametrize("kind,H,KV,D", SHAPES)
def test_paged_lengths(S, kind, H, KV, D, mask):
    page = {128: 16, 64: 32, 80: 64, 4: 256}[D]
    log("paged %s %s heads %d/%d dim %d, pages of %d" % (mask, kind, H, KV, D, page))
    rng = np.random.default_rng(9)
    bits = sum([_tree(rng, n) for n in NEW], []) if mask == "tree" else None
    p = Paged(S, kind, H, KV, D, PAST, NEW, page=page, bits=bits, words=1 if bits else 0)
    p.run(mask)
    log("  %.3g of the bound" % p.check(mask))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_page_sizes(S, page):
    for kind in TYPES:
        p = Paged(S, kind, 4, 2, 64, [5, 700, 255, 256, 257], [1, 1, 20, 1, 3], page=page)
        p.run("causal")
        p.check("causal")


@pytest.mark.parametrize("kind", list(TYPES))
def test_tree_masks(S, kind):
    """Rows that see nothing, rows that see the context alone, bits past the rows and past the words, several words."""
    rng = np.random.default_rng(10)
    new = [70, 5, 130, 1, 1]
    past = [0, 9, 33, 0, 40]
    bits = []
    for b, n in enumerate(new):
        t = _tree(rng, n, empty=[0, n // 2] if n > 1 else [0])
        bits += [m | 1 << (n + 3) if i % 3 == 0 else m for i, m in enumerate(t)]     # a bit of no row
    p = Paged(S, kind, 6, 2, 64, past, new, bits=bits, words=3)
    p.run("tree")
    p.check("tree")
    got = host(p.out)
    assert not got[0].any() and not got[35].any() and not got[205].any()    # no key at all
    p = Paged(S, kind, 6, 2, 64, past, new, bits=bits, words=1)             # rows from 64 on are seen by none
    p.run("tree")
    p.check("tree")


@pytest.mark.parametrize("kind", list(TYPES))
def test_paged_padding_and_odd_lengths(S, kind):
    used = [0, 1, 7, -2, 40]
    p = Paged(S, kind, 4, 2, 128, [10, 100, 64, 5, 0], [4, 1, 9, 6, 33], used=used)
    for mask in ("none", "causal"):
        p.run(mask)
        p.check(mask)


@pytest.mark.parametrize("kind", list(TYPES))
def test_lengths_that_contradict(S, kind):
    """Fewer keys than rows (the first rows stand before the first key), none at all, and more than the table has."""
    p = Paged(S, kind, 4, 1, 64, [30, 20, 10, 40], [6, 6, 6, 6], kv_len=[3, 0, -7, 1000], width=3)
    p.run("causal")
    p.check("causal")


@pytest.mark.parametrize("kind", list(TYPES))
def test_pages_that_are_none(S, kind):
    """Table entries outside the pool hide their keys; a request with no page at all gives zeros."""
    import torch
    p = Paged(S, kind, 4, 2, 128, [200, 100, 330, 64], [1, 20, 2, 1], page=16)
    p.table[0, [0, 5, 12]] = [-1, p.P, p.P + 7]
    p.table[1, 7] = -9
    p.table[2, 3:20] = 2 ** 31 - 1
    p.table[3, :] = -1
    p.table_d = dev(p.table)
    for mask in ("none", "causal"):
        p.run(mask)
        p.check(mask)
    assert not host(p.out)[23].any()


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("bf16", 64), ("v16", 128), ("v16", 64), ("f32", 64)])
def test_paged_unseen_nan_and_infinity(S, kind, D):
    """What a sibling in the tree holds reaches a row in no way."""
    new, past = [12, 20], [30, 70]
    bits = [1 << i | (1 if i % 2 else 0) for i in range(12)] + [1 << i for i in range(20)]
    p = Paged(S, kind, 4, 2, D, past, new, bits=bits, words=1)
    inf, nan = float("inf"), float("nan")
    for b, t, k, v in ((0, 30, None, inf), (0, 34, nan, None), (0, 37, None, -inf), (1, 75, None, nan), (1, 80, nan, nan)):
        page, at = p.table[b, t // 16], t % 16
        if v is not None:
            p.pool.view(p.vt)[page, 1, :, at, 3] = v
        if k is not None:
            p.pool[page, 0, :, at, 1] = k
    p.run("tree")
    got = host(p.out)
    H = 4
    nan_rows = [4, 12 + 10]                     # their own key is NaN
    fine = [i for i in range(32) if i not in nan_rows]
    assert np.isnan(got[nan_rows]).all()
    keep = got.reshape(-1, H, D)
    q = host(p.q).reshape(-1, H, D)
    pk, pv = host(p.pool[:, 0]), host(p.pool.view(p.vt)[:, 1])
    for b, s in ((0, 0), (1, 12)):
        k, v, ok = cached_rows(pk, pv, p.table[b], p.kv[b])
        rows = [i - s for i in fine if s <= i < s + new[b]]
        check(keep[s:s + new[b]], q[s:s + new[b]], k, v, sees("tree", new[b], p.kv[b], bits[s:s + new[b]]), *TYPES[kind],
              "request %d" % b, rows=rows)


@pytest.mark.parametrize("kind,H,KV,D,page", [("bf16", 8, 2, 128, 64), ("v16", 4, 4, 128, 16), ("bf16", 14, 2, 64, 256),
                                              ("f32", 4, 1, 128, 128)])
def test_long_contexts(S, kind, H, KV, D, page):
    """Long and short contexts beside each other: the keys are split over workgroups and joined."""
    p = Paged(S, kind, H, KV, D, [20000, 3, 0, 4097, 640], [1, 1, 1, 3, 2], page=page, factor=2.0)
    p.run("causal")
    p.check("causal")
    first = p.out.clone()
    p.run("causal")
    assert host(first).tobytes() == host(p.out).tobytes(), "the same call twice gives other bits"


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_many_rows_over_a_context(S, kind):
    """A further part of a prompt, and a window both ways, over a context."""
    n = 700 if kind == "bf16" else 150
    p = Paged(S, kind, 4, 2, 128, [900, 17], [n, 130], page=64)
    for mask in ("causal", "none"):
        p.run(mask)
        p.check(mask, rows=[0, 1, 31, 32, 63, 64, 127, 128, 129, 149, 300, 639, 699])


def test_pool_past_32_bits(S):
    """Pages behind the first 4 GiB of a pool."""
    p = Paged(S, "bf16", 8, 8, 128, [300, 40], [1, 3], page=256, first_page=4500, spare=2)
    assert p.pool.numel() * 2 > (1 << 32) and (p.table[p.table >= 0] >= 4500).all()
    p.run("causal")
    p.check("causal")


def test_many_requests(S):
    """More requests than a workgroup has threads, most of them empty."""
    rng = np.random.default_rng(12)
    past = rng.integers(0, 90, size=700).tolist()
    new = (rng.random(700) < 0.3).astype(int).tolist()
    for kind in ("bf16", "f32"):
        p = Paged(S, kind, 2, 1, 64, past, new)
        p.run("causal")
        p.check("causal")


def test_prompt_and_pages_agree_with_each_other(S):
    """A prompt's rows stored in pages, then attended to as a whole and in two parts: the prompt's own output."""
    import torch
    for kind in TYPES:
        pr = Prompt(S, kind, 4, 2, 128, [150], pad=0)
        pr.run(S.SEER_MASK_CAUSAL)
        pr.check("causal")
        pages = S.seer_page_desc(32, 6, 5)
        pool = torch.full((6, 2, 2, 32, 128), float("nan"), dtype=pr.qt, device="cuda")
        table = dev(np.array([[4, 0, 5, 2, 1]]))
        slots = np.array([[4, 0, 5, 2, 1][t // 32] * 32 + t % 32 for t in range(150)])
        S.seer_kv_store(pr.desc, pages, pr.k, pr.k.stride(0), pr.v, pr.v.stride(0), 150, dev(slots), pool)
        out = torch.zeros(150, 4 * 128, dtype=pr.qt, device="cuda")
        whole = pr.out[:150, :512].float()
        for first in (0, 90, 149):
            n = 150 - first
            S.seer_attn_paged(pr.desc, pages, S.SEER_MASK_CAUSAL, pr.q[first:], pr.q.stride(0), out, 512, n,
                              dev(np.array([0, n])), None, 1, pool, table, dev(np.array([150])), None, 0, pr.ws)
            diff = (out[:n].float() - whole[first:]).abs().max().item()
            assert diff <= (1e-5 if kind == "f32" else 0.05), (kind, first, diff)


@pytest.mark.parametrize("kind", list(TYPES))
def test_on_another_stream_and_recorded(S, kind):
    """Two recorded calls of different sizes on one workspace and one stream, replayed between eager calls; an eager
    call on another stream with a workspace of its own."""
    import torch
    from paper_2607_14557_amd.runner import record
    a = Paged(S, kind, 8, 2, 128, [3000, 17, 500], [1, 1, 1], page=64, seed=2)
    b = Paged(S, kind, 8, 2, 128, [700, 9], [30, 2], page=64, seed=3)
    pr = Prompt(S, kind, 8, 2, 128, [130, 40], seed=4)
    ws = workspace(S, a.desc, max(a.rows, b.rows, pr.rows), 3)
    torch.cuda.synchronize()
    ref = {}
    for name, x, m in (("a", a, "causal"), ("b", b, "none")):
        x.run(m)
        x.check(m)
        ref[name] = x.out.clone()
    pr.run(S.SEER_MASK_CAUSAL)
    pr.check("causal")
    ref["p"] = pr.out.clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    ga = record(lambda: a.run("causal", stream=st, ws=ws), st)
    gb = record(lambda: (b.run("none", stream=st, ws=ws), pr.run(S.SEER_MASK_CAUSAL, stream=st)), st)
    for i in range(4):
        for x in (a, b, pr):
            x.out.fill_(9.0)
        st.wait_stream(torch.cuda.current_stream())
        ga.replay(st)
        gb.replay(st)
        torch.cuda.current_stream().wait_stream(st)
        for name, x in (("a", a), ("b", b), ("p", pr)):
            assert host(x.out).tobytes() == host(ref[name]).tobytes(), (i, name)
        a.run("causal")                              # eager, its own workspace, the default stream
        torch.cuda.synchronize()
        assert host(a.out).tobytes() == host(ref["a"]).tobytes()
    ga.close()
    gb.close()


@pytest.mark.parametrize("kind,H,KV,mask", [("bf16", 32, 32, "causal"), ("v16", 14, 7, "causal"), ("bf16", 32, 8, "none")])
def test_several_rounds_of_tiles(S, kind, H, KV, mask):
    """More tiles of 128 rows than run at once: the requests by their length, ties, empty ones, a request of 65 and more."""
    lens = [700, 0, 300, 300, 129, 1, 1300, 640] if KV == 32 else [900, 2100, 0, 1500, 64, 2100, 128, 1, 777, 3000]
    p = Prompt(S, kind, H, KV, 128, lens)
    p.run(S.SEER_MASK_CAUSAL if mask == "causal" else S.SEER_MASK_NONE)
    p.check(mask, rows=[0, 127, 128, 299, 640, 1299, 2099])


def _set_keys(p, k, at=None, v=None):
    """Every key of request 0 becomes k, but key `at` zeros with the value v."""
    import torch
    pool = p.pool.view(p.P, 2, p.shape[1], p.page, p.shape[2])
    for t in range(p.kv[0]):
        page, i = p.table[0, t // p.page], t % p.page
        pool[page, 0, :, i] = torch.zeros_like(k) if t == at else k
        if t == at:
            pool.view(p.vt)[page, 1, :, i] = v


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("kind", list(TYPES))
def test_a_large_value_with_no_weight(S, kind, new):
    """A value near the type's end whose key lies 120 below the others in score."""
    p = Paged(S, kind, 1, 1, 64, [200], [new])
    p.q.copy_(p.q[:1].expand_as(p.q))
    _set_keys(p, p.q[0] * (120 * 8 / p.q[0].float().square().sum()).to(p.qt), at=7, v=60000.0 if kind == "v16" else 3e38)
    p.run("none")
    p.check("none")


@pytest.mark.parametrize("kind", list(TYPES))
def test_many_small_weights(S, kind):
    """A first key with 2^23.5 times the weight of each of the 100,000 that follow, and no value."""
    p = Paged(S, kind, 1, 1, 64, [100000], [1], page=256)
    q = p.q[0].float()
    p.pool[:, 0] = 0
    page = p.table[0, 0]
    p.pool[page, 0, :, 0] = (q * (23.5 * np.log(2) * 8 / q.square().sum())).to(p.qt)
    p.pool.view(p.vt)[page, 1, :, 0] = 0
    used = dev(np.unique(p.table[p.table >= 0]))
    p.pool.view(p.vt)[used.long(), 1] = p.pool.view(p.vt)[used.long(), 1].abs().clamp(max=4)
    p.run("none")
    p.check("none")


@pytest.mark.parametrize("past", [[2999], [1216, 1152], [3000, 900, 7, 0], [12000, 4100], [64 * 512, 64]])
@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 16, 8, 128), ("v16", 14, 2, 64), ("f32", 8, 2, 64), ("bf16", 40, 1, 128)])
def test_few_tiles_of_many_keys(S, kind, H, KV, D, past):
    """Keys in runs, a run a workgroup, and lines that cross from tile to tile."""
    for new, mask in ((1, "causal"), (3, "none")):
        p = Paged(S, kind, H, KV, D, past, [new] * len(past), page=64)
        p.run(mask)
        p.check(mask)
