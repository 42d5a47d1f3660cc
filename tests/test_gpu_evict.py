"""Eviction from the cache against the oracle, exactly: choices per head and shared, protected tokens, ties, NaN and
infinite weights, lengths around what a workgroup takes at once, pages that are none, marks in place and apart."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from gqa_util import desc, torch_types
from oracle.budget import choose, moves

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


class Cache:
    """Requests of lens[b] tokens; K and V hold the place and head that a row comes from."""

    def __init__(self, S, kind, KV, D, lens, page=16, seed=1, width=None, weight=None, order="places"):
        import torch
        self.S, self.kind, self.KV, self.D, self.lens, self.page = S, kind, KV, D, lens, page
        r = np.random.default_rng(seed)
        need = [-(-n // page) for n in lens]
        self.B, self.W, self.P = len(lens), width or max(max(need), 1), sum(need) + 3
        ids, at = r.permutation(self.P), 0
        self.table = np.full((self.B, self.W), -1)
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        kt, vt = torch_types(kind)
        shape = (self.P, KV, page)
        # rows that tell where they come from: exact in bf16 piece by piece
        code = np.arange(self.P * KV * page).reshape(shape)
        rows = np.zeros(shape + (D,))
        for i in range(4):
            rows[..., i] = code >> 7 * i & 127
        rows[..., 4:] = r.integers(-100, 100, shape + (D - 4,))
        self.pool = torch.zeros((self.P, 2, KV, page, D), dtype=kt, device="cuda")
        self.pool[:, 0] = torch.from_numpy(rows).to(kt).cuda()
        self.pool.view(vt)[:, 1] = torch.from_numpy(rows + 1).to(vt).cuda()
        self.weight = (weight(r, shape) if weight else r.standard_exponential(shape)).astype(np.float32)
        self.number = np.full(shape, -9)
        for b, n in enumerate(lens):
            for h in range(KV):
                to = np.arange(n) if order == "places" else r.permutation(n)
                if order == "same" and h:
                    to = first
                first = to
                for j in range(n):
                    self.number[self.table[b, j // page], h, j % page] = to[j]
        self.desc, self.pages = desc(S, kind, KV, KV, D), S.seer_page_desc(page, self.P, self.W)
        n = S.seer_kv_evict_workspace_bytes(self.desc, self.pages, self.B)
        self.ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")

    def upload(self):
        import torch
        self.k, self.v = host(self.pool[:, 0]), host(self.pool.view(torch_types(self.kind)[1])[:, 1])
        self.got = self.pool.clone()
        self.w, self.n = torch.from_numpy(self.weight).cuda(), dev(self.number)
        self.kept = dev(np.full(self.B, 77))

    def run(self, budget, first=0, recent=0, shared=False, apart=False, seen=None, stream=None):
        import torch
        self.upload()
        self.apart, self.seen = apart, list(self.lens) if seen is None else seen
        self.wo = torch.full_like(self.w, 7.0) if apart else self.w
        self.no = torch.full_like(self.n, 7) if apart else self.n
        self.call(dev(np.array(budget)), dev(np.array(self.seen)), first, recent, shared, stream)
        self.check(budget, first, recent, shared)

    def call(self, budget, seen, first, recent, shared, stream=None):
        self.S.seer_kv_evict(self.desc, self.pages, self.S.SEER_EVICT_SHARED if shared else 0, dev(np.array(self.lens)), budget,
                             seen, self.B, first, recent, dev(self.table), self.got, self.w, self.n, self.wo, self.no,
                             self.kept, self.ws, stream=stream)

    def check(self, budget, first, recent, shared):
        k, v = self.k.copy(), self.v.copy()
        w, n = (np.full(self.weight.shape, 7.0, np.float32), np.full(self.number.shape, 7)) if self.apart else \
            (self.weight.copy(), self.number.copy())
        for b, L in enumerate(self.lens):
            N = max(0, min(budget[b], L))
            at = [(int(self.table[b, j // self.page]), j % self.page) for j in range(L)]
            ok = [0 <= p < self.P for p, _ in at]
            worth = lambda h: [self.weight[p, h, s] if o else -np.inf for (p, s), o in zip(at, ok)]
            age = lambda h: [self.number[p, h, s] if o else None for (p, s), o in zip(at, ok)]
            for h in range(self.KV):
                if shared:
                    with np.errstate(over="ignore"):          # sums past fp32 are infinities
                        by = [np.float32(np.sum(self.weight[p, :, s].astype(np.float64))) if o else -np.inf
                              for (p, s), o in zip(at, ok)]
                    number = age(0)
                else:
                    by, number = worth(h), age(h)
                # a token without a page is lighter than any weight and not protected
                lost = [j for j in range(L) if not ok[j]]
                live = [j for j in range(L) if ok[j]]
                order = choose([by[j] for j in live], [number[j] for j in live], len(live), first, recent, self.seen[b])
                stay = ([live[i] for i in order] + lost)[:N]
                src, dst = moves(stay, N)
                come = dict(zip(dst, src))
                for j in range(N):
                    i = come.get(j, j)
                    if not ok[i] or not ok[j] or (i == j and not self.apart):
                        continue
                    (p, s), (fp, fs) = at[j], at[i]
                    w[p, h, s], n[p, h, s] = self.weight[fp, h, fs], self.number[fp, h, fs]
                    if i != j:
                        k[p, h, s], v[p, h, s] = self.k[fp, h, fs], self.v[fp, h, fs]
        assert host(self.kept).tolist() == [max(0, min(m, L)) for m, L in zip(budget, self.lens)]
        assert np.array_equal(host(self.no), n)
        assert np.array_equal(host(self.wo), w.astype(np.float64), equal_nan=True)
        assert np.array_equal(host(self.got[:, 0]), k), "keys"
        assert np.array_equal(host(self.got.view(torch_types(self.kind)[1])[:, 1]), v), "values"


LENS = [0, 1, 2, 5, 16, 17, 64, 100, 130, 255, 256, 257, 300]
KINDS = [("bf16", 2, 128), ("v16", 3, 64), ("f32", 2, 4), ("f32", 1, 80)]


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("kind,KV,D", KINDS)
def test_lengths(S, kind, KV, D, shared, apart):
    log("%s %d heads dim %d shared %s apart %s" % (kind, KV, D, shared, apart))
    for order in ("places", "same" if shared else "mixed"):
        c = Cache(S, kind, KV, D, LENS, order=order)
        c.run([max(0, n - 1) for n in LENS], 1, 3, shared, apart)
        c.run([n // 2 for n in LENS], 2, 5, shared, apart)
        c.run([1] * len(LENS), 0, 0, shared, apart)
        c.run([0] * len(LENS), 4, 4, shared, apart)
        c.run(LENS, 4, 4, shared, apart)
        c.run([-5, 9, 9, 9, 1000, 3, 60, 60, 60, 60, 60, 60, 60], 4, 4, shared, apart)


def test_protected(S):
    """More protected tokens than the budget, all of them, and a count of tokens far from their number in the cache."""
    for order in ("places", "mixed"):
        c = Cache(S, "bf16", 2, 64, [40, 50, 300], order=order)
        c.run([10, 10, 100], 8, 8)
        c.run([10, 10, 100], 30, 30)
        c.run([10, 10, 100], 1000, 0)
        c.run([10, 10, 100], 0, 2 ** 31 - 1)
        c.run([10, 10, 100], 2, 5, seen=[1000, 45, 2 ** 31 - 1])
        c.run([10, 10, 100], 2, 5, seen=[0, -5, -2 ** 31])


@pytest.mark.parametrize("shared", [False, True])
def test_ties_and_odd_weights(S, shared):
    """Equal weights, both zeros, negative ones, infinities and NaN: the lower place of equal ones stays."""
    def few(r, shape):
        return r.choice([0.0, -0.0, 1.0, 1.0, 2.5, -1.0], shape)

    def odd(r, shape):
        return r.choice([0.0, 1e-45, -1e-45, 3e38, -3e38, np.inf, np.inf if shared else -np.inf, np.nan, 1.0], shape)

    def near(r, shape):                            # neighbours in every byte of the order
        return np.float32(1.0) + r.integers(0, 4, shape) * np.float32(2.0 ** -23)

    def none(r, shape):
        return np.zeros(shape)

    for weight in (few, odd, near, none):
        for KV in (1, 2):
            c = Cache(S, "bf16", KV, 64, [1, 30, 200, 333], weight=weight, order="same")
            c.run([1, 12, 80, 150], 2, 3, shared)
            c.run([1, 29, 199, 5], 0, 0, shared, apart=True)


@pytest.mark.parametrize("kind,KV,D,page", [("bf16", 1, 64, 256), ("f32", 2, 4, 32), ("v16", 2, 64, 128)])
def test_long(S, kind, KV, D, page):
    """Places of several stretches of a workgroup, beside short ones."""
    lens = [1023, 1024, 1025, 2100, 7000, 3]
    for shared in (False, True):
        c = Cache(S, kind, KV, D, lens, page=page, order="same")
        c.run([n - 1 for n in lens], 2, 40, shared)
        c.run([600] * 6, 2, 40, shared, apart=True)
        c.run([5000] * 6, 0, 700, shared)


def test_very_long(S):
    """More places than any one stretch or LDS holds."""
    c = Cache(S, "f32", 1, 4, [70000], page=256, order="same")
    c.run([3000], 4, 100)
    c.run([69000], 4, 100, apart=True)


def test_many_requests(S):
    r = np.random.default_rng(2)
    lens = [int(x) for x in r.integers(0, 60, 600)]
    c = Cache(S, "f32", 2, 4, lens)
    c.run([int(x) for x in r.integers(0, 60, 600)], 1, 2)
    c.run([int(x) for x in r.integers(0, 60, 600)], 1, 2, shared=True)


def test_pages_that_are_none(S):
    """Their tokens go first, nothing is read from them or written to them."""
    for shared in (False, True):
        c = Cache(S, "bf16", 2, 64, [100, 60], width=9)
        c.table[0, 1], c.table[0, 6], c.table[1, 3] = -1, c.P, 1 << 30
        c.run([70, 50], 2, 20, shared)
        c.run([99, 10], 2, 20, shared, apart=True)
        c.run([5, 59], 0, 0, shared)


def test_repeated_and_recorded(S):
    """Marks apart: the call can be made again; and replayed with other weights."""
    import torch
    from paper_2607_14557_amd.runner import record
    c = Cache(S, "bf16", 2, 64, [100, 333], order="mixed")
    c.run([60, 200], 2, 9, apart=True)
    budget, seen = dev(np.array([60, 200])), dev(np.array(c.seen))
    lens, table = dev(np.array(c.lens)), dev(c.table)
    call = lambda s=None: S.seer_kv_evict(c.desc, c.pages, 0, lens, budget, seen, 2, 2, 9, table, c.got, c.w, c.n, c.wo, c.no,
                                          c.kept, c.ws, stream=s)
    for _ in range(3):
        call()
        c.check([60, 200], 2, 9, False)
    st = torch.cuda.Stream()
    graph = record(lambda: call(st), st)
    r = np.random.default_rng(8)
    for i in range(4):
        c.weight = r.standard_exponential(c.weight.shape).astype(np.float32)
        c.w.copy_(torch.from_numpy(c.weight))
        c.got.copy_(c.pool)
        c.wo.fill_(7.0)
        c.no.fill_(7)
        torch.cuda.synchronize()
        graph.replay(st)
        torch.cuda.synchronize()
        c.check([60, 200], 2, 9, False)
