"""Attention weights and eviction where another form of the kernels is taken: by the number of lists and their length,
of requests, rows and heads; cases at the ends of what a call may be; two recordings with one workspace."""
import numpy as np
import pytest

from gpu_util import dev, log
from oracle.budget import choose, moves
from test_gpu_attn_weights import Call, _bits, _gen, _normal
from test_gpu_evict import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


@pytest.mark.parametrize("shared,lists", [(False, 8), (False, 300), (False, 520), (True, 270), (True, 3)])
@pytest.mark.parametrize("most", [150, 2500, 8300])
def test_lists(S, shared, lists, most):
    """Few and many lists, whose row of the table is short, longer and longest: each kernel of the choice, with the moves in
    the same launch and in one of their own."""
    log("%d lists of up to %d places, shared %s" % (lists, most, shared))
    heads = 1 if shared else 4
    r = np.random.default_rng(lists + most)
    lens = [most] + [int(x) for x in r.integers(0, 90, lists // heads - 1)]
    c = Cache(S, "f32", 4 if shared else heads, 4, lens, page=64, order="same")
    for apart in (False, True):
        c.run([int(n * f) for n, f in zip(lens, r.random(len(lens)))], 2, 7, shared, apart)


@pytest.mark.parametrize("places", [3000, 9000, 20000])
@pytest.mark.parametrize("shared", [False, True])
def test_wide_tables(S, places, shared):
    """Lists of which all but one are much shorter than their row of the table, few and many of them."""
    r = np.random.default_rng(places)
    for n in (4, 140):
        lens = [2047, 2048, 2049, places - 40][: 4 if n == 4 else 3] + [int(x) for x in r.integers(0, 300, n)]
        c = Cache(S, "f32", 4, 4, lens, page=64, order="same", width=-(-places // 64))
        c.run([int(m * f) for m, f in zip(lens, r.random(len(lens)))], 2, 7, shared)
        c.run([max(0, m - 1) for m in lens], 2, 7, shared, True)


@pytest.mark.parametrize("kind,KV,D", [("bf16", 9, 64), ("bf16", 8, 128), ("f32", 11, 4), ("f32", 8, 80)])
def test_heads_of_lists_that_move_themselves(S, kind, KV, D):
    r = np.random.default_rng(KV)
    lens = [int(x) for x in r.integers(0, 70, 520 // KV + 1)]
    c = Cache(S, kind, KV, D, lens)
    c.run([n // 2 for n in lens], 1, 3)
    c.run([n - 1 for n in lens], 0, 0, apart=True)


@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 16, 8, 128), ("bf16", 8, 8, 64), ("bf16", 16, 16, 64), ("f32", 16, 8, 4)])
@pytest.mark.parametrize("mask", ["causal", "none", "tree"])
def test_heads_by_eights(S, kind, H, KV, D, mask):
    """Heads that divide by the dies, on tiles and with scores kept."""
    for past, lens in (([0, 130, 70], [150, 1, 65]), ([300, 0, 65], [1, 2, 1])):
        c = Call(S, kind, H, KV, D, past, lens, bits=_bits(lens) if mask == "tree" else None)
        c.run(mask)
        c.check(mask)


@pytest.mark.parametrize("rows", [8, 9, 17, 32, 33, 64, 65])
def test_rows_of_a_tile(S, rows):
    """Requests of one group of a tile's rows, of some, of all, and of a row more; all with keys in three tiles."""
    for mask in ("causal", "none", "tree"):
        lens = [rows, 1, 2]
        c = Call(S, "bf16", 1, 1, 64, [140, 40, 0], lens, bits=_bits(lens) if mask == "tree" else None)
        c.run(mask)
        c.check(mask)
        c = Call(S, "bf16", 4, 1, 128, [140, 40, 0], lens, bits=_bits(lens) if mask == "tree" else None)
        c.run(mask, last=8)
        c.check(mask, last=8)


@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 16, 1, 128), ("v16", 14, 2, 64), ("bf16", 8, 8, 64)])
@pytest.mark.parametrize("mask", ["causal", "none", "tree"])
def test_rows_in_parts(S, kind, H, KV, D, mask):
    """Many rows over few keys: each tile of keys adds its rows up in parts, some of which have none."""
    for past, lens, last in (([300], [100], 0), ([70, 0, 5], [3, 130, 0], 0), ([0, 200], [150, 90], 70), ([0], [600], 0)):
        if KV == 8:
            past, lens = past[:1], [8 * n for n in lens[:1]]
        if mask == "tree" and max(lens) > 200:
            continue
        c = Call(S, kind, H, KV, D, past, lens, bits=_bits(lens) if mask == "tree" else None, page=64)
        for decay in (1.0, 0.0):
            c.run(mask, last=last, decay=decay)
            c.check(mask, last=last, decay=decay)


@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 4, 1, 128), ("bf16", 8, 8, 64), ("bf16", 16, 1, 64)])
def test_trees_across_words(S, kind, H, KV, D):
    """Trees whose first key lies at several places of a tile of 32 keys, and whose rows pass a word of 64."""
    for past in (0, 1, 31, 32, 33, 63, 64, 95, 100, 127):
        lens = [70, 1, 9, 2]
        c = Call(S, kind, H, KV, D, [past, past + 1, past, 0], lens, bits=_bits(lens, past))
        c.run("tree")
        c.check("tree")
        c.run("tree", last=2)
        c.check("tree", last=2)


def test_most_requests(S):
    """As many as a call takes, most of one token: the requests' line is at its longest beside the scores' tiles."""
    r = np.random.default_rng(9)
    lens = [int(x) for x in r.integers(0, 2, 4096)]
    past = [int(x) for x in r.integers(0, 20, 4096)]
    for kind, D in (("bf16", 128), ("f32", 4)):
        c = Call(S, kind, 2, 1, D, past, lens)
        c.run("causal")
        c.check("causal", requests=set(range(0, 4096, 61)))


def test_offsets_that_fall(S):
    """Row offsets that are none: no weight is written, and nothing past the workspace."""
    import torch
    c = Call(S, "bf16", 4, 2, 64, [40, 30, 20], [9, 9, 9])
    c.cu_d = dev(np.array([0, 18, 0, 27]))
    tail = torch.full((4096,), 0x5a, dtype=torch.uint8, device="cuda")
    need = c.ws.numel()
    whole = torch.cat([c.ws, tail])
    c.run("causal", ws=whole[:need])
    torch.cuda.synchronize()
    assert (c.weight == 7.0).all() and (whole[need:] == 0x5a).all()


def test_far_pages(S):
    """Pages whose rows and marks lie past 2^31 elements of the pool: weights, then the eviction."""
    import torch
    H, KV, D, page = 2, 1, 128, 256
    P = (1 << 31) // (2 * KV * page * D) + 40              # pages of which the last lie past 2^31 elements
    c = Call(S, "bf16", H, KV, D, [700], [9], page=page)
    small, ids = c.pool, [int(x) for x in c.table[0]]
    far = [P - 1 - i for i in range(len(ids))]
    pool = torch.empty(P, 2, KV, page, D, dtype=torch.bfloat16, device="cuda")
    weight = torch.full((P, KV, page), 7.0, device="cuda")
    number = torch.full((P, KV, page), -1, dtype=torch.int32, device="cuda")
    prev = torch.zeros(P, KV, page, device="cuda")
    small[:, 1] = 1.0
    for i, f in zip(ids, far):
        pool[f], prev[f] = small[i], c.prev[i]
        number[f] = torch.arange(page, dtype=torch.int32, device="cuda") + 1000 * (P - f)
    c.run("causal")
    want = c.weight.clone()
    c.check("causal")
    pages, table = S.seer_page_desc(page, P, len(far)), dev(np.array([far]))
    ws = torch.empty(S.seer_attn_weights_workspace_bytes(c.desc, pages, c.rows, 1), dtype=torch.uint8, device="cuda")
    S.seer_attn_weights(c.desc, pages, 1, c.q, c.q.stride(0), c.rows, c.cu_d, None, 1, 0, pool, table, c.kv_d, None, 0, 1.0, prev,
                        weight, ws)
    for i, f in zip(ids, far):
        assert torch.equal(weight[f], want[i])
    L, N = 709, 300
    before = [pool[f].clone() for f in far]
    at = [(j // page, j % page) for j in range(L)]
    w = [float(weight[far[p], 0, s]) for p, s in at]
    marks = [int(number[far[p], 0, s]) for p, s in at]
    ws = torch.empty(S.seer_kv_evict_workspace_bytes(c.desc, pages, 1), dtype=torch.uint8, device="cuda")
    S.seer_kv_evict(c.desc, pages, 0, dev(np.array([L])), dev(np.array([N])), dev(np.array([10 ** 6])), 1, 0, 0, table, pool, weight,
                    number, weight, number, dev(np.array([0])), ws)
    src, dst = moves(choose(np.array(w, np.float32), marks, N, 0, 0, 10 ** 6), N)
    for s, d in zip(src, dst):
        (fp, fs), (tp, ts) = at[s], at[d]
        assert torch.equal(pool[far[tp], :, 0, ts], before[fp][:, 0, fs])
        assert int(number[far[tp], 0, ts]) == marks[s] and float(weight[far[tp], 0, ts]) == w[s]


def test_two_recordings_one_workspace(S):
    """Weights and eviction recorded twice with the same workspaces, replayed in turn on one stream, with eager calls
    between."""
    import torch
    from paper_2607_14557_amd.runner import record
    a, b = Call(S, "bf16", 8, 2, 128, [900, 30], [3, 50], seed=1), Call(S, "bf16", 8, 2, 128, [400, 64], [1, 90], seed=2)
    ws = a.ws if a.ws.numel() >= b.ws.numel() else b.ws
    ea, eb = (Cache(S, "bf16", 2, 64, [100, 333], seed=s, order="mixed") for s in (3, 4))
    ews = ea.ws
    st = torch.cuda.Stream()
    args = {}
    for e in (ea, eb):
        e.run([60, 200], 2, 9, apart=True)
        e.ws = ews
        args[id(e)] = (dev(np.array([60, 200])), dev(np.array(e.seen)), dev(np.array(e.lens)), dev(e.table))

    def cut(e, s=None):
        budget, seen, lens, table = args[id(e)]
        S.seer_kv_evict(e.desc, e.pages, 0, lens, budget, seen, 2, 2, 9, table, e.got, e.w, e.n, e.wo, e.no, e.kept, ews, stream=s)

    def step(c, e, s):
        c.run("causal", stream=s, ws=ws)
        cut(e, s)

    graphs = [record(lambda: step(a, ea, st), st), record(lambda: step(b, eb, st), st)]
    for i in range(4):
        for c, e in ((a, ea), (b, eb)):
            c.q.copy_(_normal(_gen(40 + i), *c.q.shape))
            c.weight.fill_(7.0)
            e.got.copy_(e.pool)
            e.wo.fill_(7.0)
            e.no.fill_(7)
        torch.cuda.synchronize()
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay(st)
        torch.cuda.synchronize()
        for c, e in ((a, ea), (b, eb)):
            c.check("causal")
            e.check([60, 200], 2, 9, False)
        a.run("causal", ws=ws)
        cut(eb)
        torch.cuda.synchronize()
