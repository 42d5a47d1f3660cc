"""The operators of a cache within a budget together, as a serving program uses them (BudgetCache): prompts, single
tokens, trees of which a part is taken, evictions per head and shared, the plan that gives their pages back, requests
that end and new ones in their places, eager and recorded, beside the same steps in float64 on the tokens themselves."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from gqa_util import TYPES, check, torch_types, words_of
from oracle.budget import choose, frequencies, moves, rotate, weights
from oracle.paged import pages_of, sees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


class Program:
    """A cache of two layers beside its tokens, per request and head: keys as they are stored, values, weights, numbers."""

    def __init__(self, S, kind, H=4, KV=2, D=64, B=4, page=16, n_pages=40, max_len=160, rows=200):
        import torch
        from paper_2607_14557_amd.runner import BudgetCache
        self.S, self.kind, self.shape, self.B, self.rows = S, kind, (H, KV, D), B, rows
        rope = S.seer_rope_desc(S.SEER_ROPE_PAIRS, 48, S.SEER_ROPE_BANDS, 64, 10000.0, 4.0, 1.0, 4.0, 0.0)
        self.freq = frequencies(48, 10000.0, "bands", 4.0, 1.0, 4.0, 64)
        self.c = BudgetCache(H, KV, D, 2, n_pages, page, B, max_len, rows, rope=rope, dtype="f32" if kind == "f32" else "bf16",
                             v_f16=kind == "v16")
        for p in self.c.pools:
            p.fill_(float("nan"))
            p.view(torch_types(kind)[1])[:, 1] = float("nan")
        self.tokens = [[dict(k=np.zeros((0, KV, D)), v=np.zeros((0, KV, D)), w=np.zeros((0, KV)), n=np.zeros((0, KV), int))
                        for _ in range(B)] for _ in range(2)]
        self.seen = [0] * B
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(3)
        self.page, self.n_pages = page, n_pages

    def held(self):
        return [len(t["k"]) for t in self.tokens[0]]

    def step(self, lens, keep=None, base=None, mask="causal", bits=None, decay=1.0, last=0):
        import torch
        H, KV, D = self.shape
        qt, vt = torch_types(self.kind)
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(int)
        T, cu_d, m = int(cu[-1]), dev(cu), dict(none=0, causal=1, tree=2)[mask]
        bits_d = None
        if bits is not None:
            bits_d = torch.zeros(self.rows, 1, dtype=torch.int64, device="cuda")
            bits_d[:T] = torch.from_numpy(words_of(bits, 1)).cuda()
        opt = lambda x: None if x is None else dev(np.array(x))
        slots = self.c.plan(cu_d, self.rows, opt(keep), base=opt(base))
        start = list(self.seen) if base is None else base
        normal = lambda n, t: torch.empty(self.rows, n * D, device="cuda").normal_(0, 1, generator=self.gen).to(t)
        for layer in range(2):
            q, k, v = normal(H, qt), normal(KV, qt), normal(KV, vt)
            plain_q, plain_k, out = host(q), host(k), torch.full((self.rows, H * D), 9.0, dtype=qt, device="cuda")
            self.c.store(layer, k, v, self.rows, slots, q=q)
            self.c.attend(layer, q, out, cu_d, self.rows, m, bits_d)
            self.c.weigh(layer, q, cu_d, self.rows, m, bits_d, decay=decay, last=last)
            got, turned, vh = host(out), host(q).reshape(-1, H, D), host(v).reshape(-1, KV, D)
            assert (got[T:] == 9.0).all() and np.array_equal(host(q)[T:], plain_q[T:])
            got = got.reshape(-1, H, D)
            pool, weight, number = host(self.c.pools[layer][:, 0]), host(self.c.weights[layer]), host(self.c.numbers[layer])
            table = host(self.c.table)
            for b, n in enumerate(lens):
                t, s = self.tokens[layer][b], cu[b]
                if keep is not None:
                    for name in t:
                        t[name] = t[name][:keep[b]]
                at = np.arange(start[b], start[b] + n)
                want = rotate(plain_k[s:s + n].reshape(n, KV, D), at, self.freq, "pairs")
                L = len(t["k"]) + n
                where = [(table[b, j // self.page], j % self.page) for j in range(L)]
                stored = np.array([pool[p, :, i] for p, i in where]).reshape(L, KV, D)
                # (the bounds of the rotation are held elsewhere; here that it is the right one)
                assert np.abs(stored[L - n:] - want).max(initial=0.0) <= 0.05
                assert np.array_equal(stored[:L - n], t["k"]), "layer %d request %d: older tokens" % (layer, b)
                t["k"], t["v"] = stored, np.concatenate([t["v"], vh[s:s + n]])
                t["n"] = np.concatenate([t["n"], np.repeat(at[:, None], KV, 1)]).astype(int)
                t["w"] = np.concatenate([t["w"], np.zeros((n, KV))])
                assert np.array_equal(np.array([number[p, :, i] for p, i in where]).reshape(L, KV), t["n"])
                if n:
                    c = min(n, last) if last else n
                    assert np.abs(turned[s:s + n] - rotate(plain_q[s:s + n].reshape(n, H, D), at, self.freq, "pairs")).max() <= 0.05
                    seen = sees(mask, n, L, None if bits is None else bits[s:s + n])
                    check(got[s:s + n], turned[s:s + n], t["k"], t["v"], seen, *TYPES[self.kind], "request %d" % b)
                    t["w"] = decay * t["w"] + weights(turned[s + n - c:s + n], t["k"], seen[n - c:])[0]
                    w = np.array([weight[p, :, i] for p, i in where]).reshape(L, KV)
                    # the bounds are held elsewhere; from here on the choices go by the device's own weights
                    assert np.abs(w - t["w"]).max() <= 1e-4 * (1 + t["w"].max())
                    t["w"] = w
        self.c.check()
        self.seen = [s + n for s, n in zip(start, lens)]
        assert host(self.c.lens).tolist() == self.held() and host(self.c.seen).tolist() == self.seen
        assert host(self.c.free).item() == self.n_pages - sum(pages_of(n, self.page) for n in self.held())

    def evict(self, budget, first, recent, shared=False):
        for layer in range(2):
            kept = self.c.evict(layer, dev(np.array(budget)), first, recent, shared)
            for b in range(self.B):
                t = self.tokens[layer][b]
                L = len(t["k"])
                N = min(budget[b], L)
                plans = [moves(choose(np.float32(t["w"].sum(1)) if shared else t["w"][:, h], t["n"][:, 0 if shared else h], N,
                                      first, recent, self.seen[b]), N) for h in range(self.shape[1])]
                for h, (source, hole) in enumerate(plans):
                    for name in t:
                        t[name][hole, h] = t[name][source, h]
                for name in t:
                    t[name] = t[name][:N]
        assert host(kept).tolist() == self.held()


@pytest.mark.parametrize("kind", list(TYPES))
def test_a_serving_program(S, kind):
    rng = np.random.default_rng(4)
    p = Program(S, kind)
    log("%s: prompts, of which the last rows say what is worth keeping" % kind)
    p.step([40, 1, 120, 17], last=8)
    p.evict([24, 24, 24, 24], 2, 4)
    log("single tokens, each with an eviction: the cache stays at its budget")
    for _ in range(4):
        p.step([1, 1, 1, 1], decay=0.9)
        p.evict([24, 24, 24, 24], 2, 4)
    log("trees of drafted tokens; some of them stay, their positions go on from there")
    lens, bits = [5, 7, 9, 0], []
    for n in lens:
        seen = []
        for i in range(n):
            up = int(rng.integers(-1, i)) if i else -1
            seen.append((seen[up] if up >= 0 else 0) | 1 << i)
        bits += seen
    p.step(lens, mask="tree", bits=bits)
    held, seen = p.held(), p.seen
    p.step([1, 1, 1, 1], keep=[held[0] - 2, held[1], held[2] - 9, held[3]], base=[seen[0] - 2, seen[1], seen[2] - 9, seen[3]])
    log("a window, both ways; one request ends, another takes its place")
    p.step([30, 0, 11, 2], mask="none")
    p.evict([20, 5, 0, 100], 1, 3)
    p.step([1, 3, 50, 1], base=[p.seen[0], p.seen[1], 0, p.seen[3]])
    p.step([1, 0, 1, 1])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_shared_choices(S, kind):
    p = Program(S, kind)
    p.step([60, 5, 100, 30], decay=1.0)
    p.evict([20, 20, 31, 29], 1, 5, shared=True)
    p.step([2, 1, 1, 1])
    p.evict([20, 6, 30, 8], 1, 5, shared=True)
    p.step([1, 1, 1, 1])


def test_a_refused_plan(S):
    """The cut stands, the counts too, and the same plan in smaller steps is taken."""
    p = Program(S, "bf16", n_pages=14)
    p.step([60, 5, 100, 30])
    p.evict([40, 5, 40, 30], 1, 5)
    before = host(p.c.seen).tolist()
    with pytest.raises(S.SeerError):
        p.c.plan(dev(np.array([0, 0, 0, 120, 120])), 200)
        p.c.check()
    assert host(p.c.seen).tolist() == before and (host(p.c.positions) == -1).all()
    p.step([1, 1, 1, 1])
    p.evict([16, 16, 16, 16], 1, 5)
    p.step([1, 1, 1, 1])


def test_recorded_steps(S):
    """Two decoding steps, each with its eviction, in one recording, replayed beside the same steps eagerly on a cache of
    its own."""
    import torch
    from paper_2607_14557_amd.runner import BudgetCache, record
    H, KV, D, B, rows = 8, 2, 128, 3, 4
    rope = S.seer_rope_desc(S.SEER_ROPE_HALF, 0, S.SEER_ROPE_PLAIN, 0, 10000.0, 1.0, 0.0, 0.0, 0.0)
    caches = [BudgetCache(H, KV, D, 1, 30, 16, B, 64, 64, rope=rope) for _ in range(2)]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    normal = lambda n: torch.empty(64, n * D, device="cuda").normal_(0, 1, generator=gen).to(torch.bfloat16)
    cu0, cu, budget = dev(np.array([0, 30, 31, 50])), dev(np.array([0, 1, 2, 3])), dev(np.array([20, 20, 20]))
    q, k, v = normal(H), normal(KV), normal(KV)
    outs = [torch.zeros(64, H * D, dtype=torch.bfloat16, device="cuda") for _ in caches]
    qo = [torch.zeros(64, H * D, dtype=torch.bfloat16, device="cuda") for _ in caches]

    def step(i, cu, n, stream=None):
        c = caches[i]
        slots = c.plan(cu, n, stream=stream)
        c.store(0, k, v, n, slots, stream=stream, q=q, q_out=qo[i])
        c.attend(0, qo[i], outs[i], cu, n, stream=stream)
        c.weigh(0, qo[i], cu, n, stream=stream)
        c.evict(0, budget, 1, 2, stream=stream)

    for i in range(2):
        step(i, cu0, 64)
        step(i, cu, rows)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()

    def two():
        step(0, cu, rows, st)
        step(0, cu, rows, st)

    g = record(two, st)
    for turn in range(4):
        for x, n in ((q, H), (k, KV), (v, KV)):
            x.copy_(normal(n))
        torch.cuda.synchronize()
        g.replay(st)
        step(1, cu, rows)
        step(1, cu, rows)
        torch.cuda.synchronize()
        a, b = caches
        assert torch.equal(outs[0], outs[1]) and torch.equal(a.weights[0], b.weights[0])
        assert torch.equal(a.numbers[0], b.numbers[0]) and torch.equal(a.pools[0], b.pools[0])
        assert torch.equal(a.lens, b.lens) and torch.equal(a.seen, b.seen) and torch.equal(a.free, b.free)
    caches[0].check()
    assert host(caches[0].seen).tolist() == [39, 10, 28]


def test_layer_rows(S):
    """store_layer: the layer's rows with marks, keys as the layer left them."""
    import torch
    from gpu_util import upload_weights, view_ws
    from paper_2607_14557_amd.runner import BudgetCache, SeerStack, dims_for
    from workloads.generate import round_to_dtype
    rng = np.random.default_rng(2)
    d, H, D, I = 256, 4, 64, 688
    dims = dims_for(d, H, D, I, "f32")
    W = {n: round_to_dtype(rng.standard_normal(s) * 0.02, "f32") for n, s in
         (("wq", (d, d)), ("wk", (d, d)), ("wv", (d, d)), ("wo", (d, d)), ("wg", (I, d)), ("wu", (I, d)), ("wd", (d, I)))}
    W.update(g1=np.ones(d), g2=np.ones(d))
    stack = SeerStack(dims, 1, 60)
    stack.set_layer(0, upload_weights(W, "f32"))
    cu = dev(np.array([0, 33, 50]))
    x = dev(rng.standard_normal((60, d)), "f32")
    stack.layer(0, x, torch.empty_like(x), cu, None, 2, 60)
    c = BudgetCache(H, H, D, 1, 10, 16, 2, 64, 60, dtype="f32")
    c.plan(cu, 60)
    c.store_layer(0, stack, 60)
    c.check()
    at = S.seer_layer_workspace_offsets(dims, 60)[0]
    qkv = host(view_ws(stack.workspace, at, 60, 3 * d, "f32"))
    slots = host(c.slots)[:50]
    pool, number = host(c.pools[0]), host(c.numbers[0])
    assert np.array_equal(pool[slots // 16, 0, :, slots % 16], qkv[:50, d:2 * d].reshape(50, H, D))
    assert np.array_equal(pool[slots // 16, 1, :, slots % 16], qkv[:50, 2 * d:].reshape(50, H, D))
    assert np.array_equal(number[slots // 16, :, slots % 16][:, 0], np.concatenate([np.arange(33), np.arange(17)]))
