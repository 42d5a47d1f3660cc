"""Cuts of a cache within a budget (BudgetCache) around recordings, refused plans and layers that are not cut alike,
beside the same steps made eagerly on a cache of its own."""
import numpy as np
import pytest

from gpu_util import dev, host

pytestmark = pytest.mark.gpu
H, KV, D, B, ROWS = 8, 2, 128, 3, 4


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


class Pair:
    """Two caches that take the same steps."""

    def __init__(self, S, layers=2, n_pages=60, budget=(20, 20, 20)):
        import torch
        from paper_2607_14557_amd.runner import BudgetCache
        rope = S.seer_rope_desc(S.SEER_ROPE_HALF, 0, S.SEER_ROPE_PLAIN, 0, 10000.0, 1.0, 0.0, 0.0, 0.0)
        self.caches = [BudgetCache(H, KV, D, layers, n_pages, 16, B, 96, 64, rope=rope) for _ in range(2)]
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(1)
        self.cu0, self.cu = dev(np.array([0, 30, 31, 50])), dev(np.array([0, 1, 2, 3]))
        self.budget, self.layers = dev(np.array(budget)), range(layers)
        zeros = lambda n: torch.zeros(64, n * D, dtype=torch.bfloat16, device="cuda")
        self.q, self.k, self.v = zeros(H), zeros(KV), zeros(KV)
        self.outs, self.qo = [zeros(H) for _ in self.caches], [zeros(H) for _ in self.caches]
        self.draw()

    def draw(self):
        import torch
        for x in (self.q, self.k, self.v):
            x.copy_(torch.empty(x.shape, device="cuda").normal_(0, 1, generator=self.gen).to(x.dtype))
        torch.cuda.synchronize()

    def step(self, i, cu, n, cut=True, stream=None):
        c = self.caches[i]
        slots = c.plan(cu, n, stream=stream)
        for layer in self.layers:
            c.store(layer, self.k, self.v, n, slots, stream=stream, q=self.q, q_out=self.qo[i])
            c.attend(layer, self.qo[i], self.outs[i], cu, n, stream=stream)
            c.weigh(layer, self.qo[i], cu, n, stream=stream)
        if cut:
            self.cut(i, stream)

    def cut(self, i, stream=None):
        for layer in self.layers:
            self.caches[i].evict(layer, self.budget, 1, 2, stream=stream)

    def same(self, what=""):
        import torch
        torch.cuda.synchronize()
        a, b = self.caches
        assert torch.equal(a.lens, b.lens) and torch.equal(a.seen, b.seen) and torch.equal(a.free, b.free), what
        assert torch.equal(self.outs[0], self.outs[1]) and torch.equal(a.kept, b.kept), what
        for x, y in ((a.weights, b.weights), (a.numbers, b.numbers), (a.pools, b.pools)):
            assert all(torch.equal(s, t) for s, t in zip(x, y)), what


@pytest.mark.parametrize("cut_before", [False, True])
def test_recorded_from_either_state(S, cut_before):
    """Two decoding steps, each with its cut, recorded behind a prompt that is cut or not: the first replay goes on from
    the prompt, the later ones from the replay before, with eager steps and steps without a cut between."""
    import torch
    from paper_2607_14557_amd.runner import record
    p = Pair(S)
    for i in range(2):
        p.step(i, p.cu0, 64, cut_before)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()

    def two():
        for _ in range(2):
            p.step(0, p.cu, ROWS, stream=st)

    g = record(two, st)
    for turn in range(5):
        p.draw()
        g.replay(st)
        torch.cuda.synchronize()
        for _ in range(2):
            p.step(1, p.cu, ROWS)
        p.same("replay %d" % turn)
        if turn == 2:                                # eager steps between, an even number of plans
            for i in range(2):
                p.step(i, p.cu, ROWS, cut=False)
                p.step(i, p.cu, ROWS, cut=False)
            p.same("eager steps")
    for c in p.caches:
        c.check()
    assert host(p.caches[0].lens).tolist() == [21, 13, 21]        # the budget and the step's row


def test_eager_behind_a_recording(S):
    """A recording of which nothing has run changes nothing; a recorded cut counts for the eager plan behind its replay,
    and only there."""
    import torch
    from paper_2607_14557_amd.runner import record
    p = Pair(S)
    for i in range(2):
        p.step(i, p.cu0, 64, cut=False)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    g = record(lambda: p.cut(0, st), st)
    for i in range(2):                                # nothing was cut
        p.step(i, p.cu, ROWS, cut=False)
        p.step(i, p.cu, ROWS, cut=False)
    p.same("before the first replay")
    assert host(p.caches[0].lens).tolist() == [32, 3, 21]
    for turn in range(3):
        p.draw()
        torch.cuda.synchronize()
        g.replay(st)
        torch.cuda.synchronize()
        p.cut(1)
        for i in range(2):
            p.step(i, p.cu, ROWS, cut=False)
            p.step(i, p.cu, ROWS, cut=False)
        p.same("turn %d" % turn)
        assert host(p.caches[0].lens).tolist()[0] == 22
    for c in p.caches:
        c.check()


def test_row_positions_kept(S):
    """kept becomes the plan's lengths, and stays where the plan was refused."""
    import torch
    for n in (1, 3, 300):
        cu, seen, kv = dev(np.arange(n + 1)), dev(np.arange(n) * 5), dev(np.arange(n) + 9)
        for status, rows in ((0, n + 3), (4, n + 3), (0, 0)):
            kept, nxt, pos = dev(np.full(n, 77)), dev(np.full(n, 77)), dev(np.full(n + 3, 77))
            S.seer_row_positions(cu, None, n, seen, None, dev(np.array([status])), rows, pos, nxt, kv_len=kv, kept=kept)
            assert host(kept).tolist() == ([77] * n if status else host(kv).tolist())
            assert host(nxt).tolist() == [5 * i + (0 if status else 1) for i in range(n)]


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("long", [1, 40, 150])
def test_layers_cut_apart(S, shared, long):
    """Layers cut to different lengths: each keeps its heaviest tokens, no more than the others keep; the plan behind them
    is refused, and one that keeps the least is taken, with its tokens whole in every layer."""
    import torch
    from paper_2607_14557_amd.runner import BudgetCache
    from oracle.budget import choose, moves
    n = 60 * long                                      # lists in each kernel of the choice
    c = BudgetCache(KV, KV, 64, 3, 2 * (n // 64 + 2), 64, 2, n + 64, n + 64, dtype="f32")
    rng = np.random.default_rng(3)
    rows = torch.from_numpy(rng.standard_normal((n + 5, KV * 64)).astype(np.float32)).cuda()
    c.plan(dev(np.array([0, n, n + 5])), n + 5)
    for layer in range(3):
        c.store(layer, rows, rows, n + 5)
        c.weights[layer].copy_(torch.from_numpy(rng.random(c.weights[layer].shape).astype(np.float32)))
    table = host(c.table)
    at = [[(int(table[b, j // 64]), j % 64) for j in range(L)] for b, L in ((0, n), (1, 5))]
    budgets = [[n // 2, 3], [n // 2 + 7, 3], [n // 3, 4]]
    least, want = [n, 5], []
    for layer in range(3):
        old, w = host(c.pools[layer][:, 0]), host(c.weights[layer])
        kept = c.evict(layer, dev(np.array(budgets[layer])), shared=shared)
        got = host(c.pools[layer][:, 0])
        for b in range(2):
            least[b] = min(least[b], budgets[layer][b])
            score = np.array([w[p, :, s] for p, s in at[b]])
            for h in range(KV):
                by = score.sum(1).astype(np.float32) if shared else score[:, h].astype(np.float32)
                src, dst = moves(choose(by, np.zeros(len(by), int) + 9, least[b], 0, 0, 10 ** 6), least[b])
                come = dict(zip(dst, src))
                for j in range(least[b]):
                    (p, s), (fp, fs) = at[b][j], at[b][come.get(j, j)]
                    assert np.array_equal(got[p, h, s], old[fp, h, fs]), (layer, b, h, j)
        want.append(host(kept).tolist())
    assert want == [[n // 2, 3], [-1 - n // 2, 3], [-1 - n // 3, -1 - 3]]
    cu = dev(np.array([0, 1, 2]))
    c.plan(cu, 2)
    with pytest.raises(S.SeerError, match="different lengths"):
        c.check()
    assert host(c.lens).tolist() == [n, 5] and host(c.kept).tolist() == want[2]
    c.plan(cu, 2, keep=dev(np.array(least)))
    c.check()
    assert host(c.lens).tolist() == [n // 3 + 1, 4] and host(c.kept).tolist() == [n // 3 + 1, 4]


def test_keep_more_than_was_kept(S):
    """Behind a cut, a keep above what it left is refused, though that many tokens were held; one up to it is taken."""
    p = Pair(S)
    for i in range(2):
        p.step(i, p.cu0, 64)
    a, b = p.caches
    assert host(a.lens).tolist() == [30, 1, 19] and host(a.kept).tolist() == [20, 1, 19]
    for keep in ([21, 1, 19], [30, 1, 19], [20, 2, 19]):
        a.plan(p.cu, ROWS, keep=dev(np.array(keep)))
        with pytest.raises(S.SeerError, match="keep exceeds"):
            a.check()
        assert host(a.kept).tolist() == [20, 1, 19]
    a.plan(p.cu, ROWS, keep=a.lens)                   # an even number of plans, as of the other cache: none
    with pytest.raises(S.SeerError, match="keep exceeds"):
        a.check()
    p.same("refused plans change nothing")
    for i, keep in enumerate((dev(np.array([20, 1, 19])), None)):
        p.caches[i].plan(p.cu, ROWS, keep=keep)
    p.same("as kept")
    a.plan(p.cu, ROWS, keep=dev(np.array([7, 0, 20])))      # less of the tokens that are there
    a.check()
    assert host(a.lens).tolist() == [8, 1, 21] and host(a.kept).tolist() == [8, 1, 21]


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("max_len", [96, 3000, 9000, 20000])
def test_evict_behind_a_refused_plan(S, shared, max_len):
    """Nothing is cut or moved and kept stays, by each kernel of the choice, in a table as wide as it takes."""
    import torch
    from paper_2607_14557_amd.runner import BudgetCache
    c = BudgetCache(KV, KV, 64, 2, 12, 16, 2, max_len, 200, dtype="f32")
    rows = torch.randn(200, KV * 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    budget = dev(np.array([20, 20]))

    def step(cu, weigh=False):
        c.plan(dev(np.array(cu)), 200)
        for layer in range(2):
            c.store(layer, rows, rows, 200)
            if weigh:
                c.weights[layer].uniform_(generator=torch.Generator(device="cuda").manual_seed(layer))
        for layer in range(2):
            c.evict(layer, budget, shared=shared)

    step([0, 90, 120], True)
    torch.cuda.synchronize()
    state = [x.clone() for x in c.pools + c.weights + c.numbers + [c.kept]]
    step([0, 100, 200])                                # more pages than there are
    torch.cuda.synchronize()
    for x, y in zip(state, c.pools + c.weights + c.numbers + [c.kept]):
        assert torch.equal(x, y)
    with pytest.raises(S.SeerError):                   # free pages, or a request that is too long
        c.check()
    assert host(c.kept).tolist() == [20, 20] and host(c.lens).tolist() == [90, 30]
    step([0, 1, 3])
    c.check()
    assert host(c.lens).tolist() == [21, 22] and host(c.kept).tolist() == [20, 20]


def test_recorded_steps_behind_a_refused_plan(S):
    """A recording goes on behind a plan that is refused: its cut leaves what was cut before, and the cache goes on as one
    that took only the steps that were accepted."""
    import torch
    from paper_2607_14557_amd.runner import record
    p = Pair(S, n_pages=7)                              # a step of a row each needs 2 + 1 + 2 pages, one of 20 each does not fit
    cu, wide = p.cu.clone(), dev(np.array([0, 20, 40, 60]))
    for i in range(2):
        p.step(i, p.cu0, 64)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()

    def two():
        for _ in range(2):
            slots = p.caches[0].plan(cu, 64, stream=st)
            for layer in p.layers:
                p.caches[0].store(layer, p.k, p.v, 64, slots, stream=st, q=p.q, q_out=p.qo[0])
            p.cut(0, st)

    g = record(two, st)
    for turn, fits in enumerate((True, False, False, True)):
        p.draw()
        cu.copy_(p.cu if fits else wide)
        torch.cuda.synchronize()
        g.replay(st)
        torch.cuda.synchronize()
        if not fits:
            with pytest.raises(S.SeerError, match="free pages"):
                p.caches[0].check()
            continue
        for _ in range(2):
            slots = p.caches[1].plan(p.cu, 64)
            for layer in p.layers:
                p.caches[1].store(layer, p.k, p.v, 64, slots, q=p.q, q_out=p.qo[1])
            p.cut(1)
        p.same("replay %d" % turn)
    p.caches[0].check()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("n", [60, 2400, 9000, 17000])
def test_budget_of_the_layers_before(S, shared, n):
    """kept as the budget of the next layer: cut as with a copy of it, whatever it says, in each kernel of the choice and by
    many workgroups of a request."""
    import torch
    kv, page, D = 8, 64, 4
    P = -(-n // page)
    d, pages = S.seer_attn_desc(kv, kv, D, S.SEER_DTYPE_F32, 0, 0.0), S.seer_page_desc(page, P, P)
    gen = torch.Generator(device="cuda").manual_seed(n)
    pool0 = torch.randn(P, 2, kv, page, D, device="cuda", generator=gen)
    w0 = torch.rand(P, kv, page, device="cuda", generator=gen)
    table, lens, seen = dev(np.arange(P)[None]), dev(np.array([n])), dev(np.array([n]))
    ws = torch.empty(S.seer_kv_evict_workspace_bytes(d, pages, 1), dtype=torch.uint8, device="cuda")
    flags = S.SEER_EVICT_ALIKE | (S.SEER_EVICT_SHARED if shared else 0)
    for kept0, want, left in ((n // 3, n // 3, n // 3), (-1 - n // 4, -1 - n // 4, n // 4), (n + 9, -1 - n, n), (0, 0, 0), (-1, -1, 0)):
        got = []
        for alias in (False, True):
            pool, w, number = pool0.clone(), w0.clone(), torch.zeros(P, kv, page, dtype=torch.int32, device="cuda")
            kept = dev(np.array([kept0]))
            budget = kept if alias else dev(np.array([kept0 if kept0 >= 0 else -1 - kept0]))
            S.seer_kv_evict(d, pages, flags, lens, budget, seen, 1, 0, 0, table, pool, w, number, w, number, kept, ws)
            got.append((pool, w, host(kept).tolist()))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert got[1][2] == [want] and got[0][2] == [left if kept0 == left else -1 - left], (kept0, got)


@pytest.mark.parametrize("n", [1, 3, 300, 4096])
def test_plan_of_what_is_kept(S, n):
    """With all tokens kept, or just those that are asked for, the plan is the plan; a keep above kept of one request, or a
    kept below zero as the keep, refuses it whole."""
    import torch
    r = np.random.default_rng(n)
    page, width = 16, 6
    held = r.integers(0, page * width - 3, n)
    keep = (held * r.random(n)).astype(int)
    cu = np.concatenate([[0], np.cumsum(r.integers(0, 4, n))])
    rows, need = int(cu[-1]) + 5, -(-held // page)
    P = int(need.sum()) + n
    table0, at = np.full((n, width), -1), 0
    for b in range(n):
        table0[b, :need[b]] = np.arange(at, at + need[b])
        at += need[b]
    free0 = np.full(P, -1)
    free0[:P - at] = np.arange(at, P)

    def plan(keep, kept):
        free, table, f_in, f_out = dev(free0), dev(table0), dev(np.array([P - at])), dev(np.array([0]))
        kv, slots, status, refused = dev(np.zeros(n, int)), dev(np.full(rows, 77)), dev(np.array([9])), dev(np.array([0]))
        S.seer_page_plan_latched(S.seer_page_desc(page, P, width), dev(held), dev(keep), dev(cu), None, n, rows, free, f_in, f_out,
                                 table, kv, slots, status, refused, kept=None if kept is None else dev(kept))
        return [free, table, f_out, kv, slots, status, refused]

    want = plan(keep, None)
    assert host(want[5]).item() == 0
    for kept in (held, keep, -1 - held, -1 - keep):
        assert all(torch.equal(x, y) for x, y in zip(want, plan(keep, kept)))
    one = np.flatnonzero(keep)
    if one.size:
        b = one[-1]
        for kept in (np.where(np.arange(n) == b, keep - 1, held), np.where(np.arange(n) == b, -keep, -1 - held)):
            free, table, f_out, kv, slots, status, refused = plan(keep, kept)
            assert host(status).item() == host(refused).item() == S.SEER_PAGES_INVALID and (host(slots) == -1).all()
            assert np.array_equal(host(table), table0) and np.array_equal(host(free), free0) and np.array_equal(host(kv), held)
            assert host(f_out).item() == P - at
    assert host(plan(-1 - keep, -1 - keep)[5]).item() == S.SEER_PAGES_INVALID
