"""The paged operators together, as a serving program uses them (PagedCache):
prompts, single tokens, trees of which a part is taken, windows that are cut,
requests that end and new ones in their places, eager and recorded; and the
pages beside the layer's own attention."""
import numpy as np
import pytest

from gpu_util import dev, host, log, upload_weights, view_ws
from gqa_util import TYPES, check, torch_types, words_of
from oracle.paged import pages_of, sees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


class Program:
    """A cache of one layer beside the keys and values themselves, per request."""

    def __init__(self, S, kind, H=4, KV=2, D=64, B=5, page=16, n_pages=40, max_len=200, rows=300):
        import torch
        from paper_2607_14557_amd.runner import PagedCache
        self.S, self.kind, self.shape, self.B, self.rows = S, kind, (H, KV, D), B, rows
        self.c = PagedCache(H, KV, D, 1, n_pages, page, B, max_len, rows, dtype="f32" if kind == "f32" else "bf16",
                            v_f16=kind == "v16")
        self.c.pools[0].fill_(float("nan"))
        self.c.pools[0].view(torch_types(kind)[1])[:, 1] = float("nan")
        self.k, self.v = [np.zeros((0, KV, D)) for _ in range(B)], [np.zeros((0, KV, D)) for _ in range(B)]
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(3)
        self.page, self.n_pages = page, n_pages

    def step(self, lens, keep=None, mask="causal", bits=None, used=None, prompt=False):
        """One step with lens[b] rows of each request; returns its slots (host)."""
        import torch
        H, KV, D = self.shape
        qt, vt = torch_types(self.kind)
        T = sum(lens)
        normal = lambda n, t: torch.empty(self.rows, n * D, device="cuda").normal_(0, 1, generator=self.gen).to(t)
        q, k, v = normal(H, qt), normal(KV, qt), normal(KV, vt)
        out = torch.full((self.rows, H * D), 9.0, dtype=qt, device="cuda")
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(int)
        cu_d, m = dev(cu), dict(none=0, causal=1, tree=2)[mask]
        used_d = None if used is None else dev(np.array(used))
        bits_d = None if bits is None else torch.zeros(self.rows, 1, dtype=torch.int64, device="cuda")
        if bits is not None:
            bits_d[:T] = torch.from_numpy(words_of(bits, 1)).cuda()
        slots = self.c.plan(cu_d, self.rows, None if keep is None else dev(np.array(keep)), used_d)
        self.c.store(0, k, v, self.rows, slots)
        if prompt:
            self.c.prompt(q, k, v, out, cu_d, self.rows, m, used_d)
        else:
            self.c.attend(0, q, out, cu_d, self.rows, m, bits_d, used_d)
        self.c.check()
        kh, vh = host(k).reshape(-1, KV, D), host(v).reshape(-1, KV, D)
        qh, got = host(q).reshape(-1, H, D), host(out)
        assert (got[T:] == 9.0).all()
        got = got.reshape(-1, H, D)
        real = lens if used is None else used
        for b in range(self.B):
            n, s = real[b], cu[b]
            kept = len(self.k[b]) if keep is None else keep[b]
            self.k[b] = np.concatenate([self.k[b][:kept], kh[s:s + n]])
            self.v[b] = np.concatenate([self.v[b][:kept], vh[s:s + n]])
            assert not got[s + n:s + lens[b]].any()
            if n:
                L = len(self.k[b])
                check(got[s:s + n], qh[s:s + n], self.k[b], self.v[b],
                      sees(mask, n, L, None if bits is None else bits[s:s + n]), *TYPES[self.kind], "request %d" % b)
        assert host(self.c.lens).tolist() == [len(x) for x in self.k]
        assert host(self.c.free).item() == self.n_pages - sum(pages_of(len(x), self.page) for x in self.k)
        return host(slots)


@pytest.mark.parametrize("kind", list(TYPES))
def test_a_serving_program(S, kind):
    rng = np.random.default_rng(4)
    p = Program(S, kind)
    log("%s: prompts" % kind)
    p.step([33, 1, 90, 0, 17], prompt=True)
    log("single tokens, a place that is not in use")
    for _ in range(3):
        p.step([1, 1, 1, 0, 1])
    log("trees of drafted tokens; then only some of them stay, with the next token")
    lens, bits = [5, 7, 0, 0, 9], []
    for n in lens:
        seen = []
        for i in range(n):
            up = int(rng.integers(-1, i))
            seen.append((seen[up] if up >= 0 else 0) | 1 << i)
        bits += seen
    base = [len(x) for x in p.k]
    p.step(lens, mask="tree", bits=bits)
    p.step([1, 1, 1, 0, 1], keep=[base[0] + 3, base[1], base[2], 0, base[4] + 9])
    log("a window of a denoising step, both ways, padded; cut at its boundary; run again")
    base = [len(x) for x in p.k]
    p.step([40, 30, 0, 0, 0], mask="none", used=[33, 30, 0, 0, 0])
    p.step([12, 8, 0, 0, 0], keep=base, mask="none")
    log("requests end, others take their places")
    p.step([20, 0, 0, 60, 1], keep=[0, len(p.k[1]), 0, 0, len(p.k[4])])
    p.step([1, 1, 0, 1, 1])
    log("a refused plan changes nothing: its status is raised, the lengths stay")
    with pytest.raises(S.SeerError):
        p.c.plan(dev(np.array([0, 0, 0, 250, 250, 250])), 250)      # 13 pages to a row of the table
        p.c.check()
    assert host(p.c.lens).tolist() == [len(x) for x in p.k]
    p.step([1, 1, 0, 1, 1])


def test_recorded_steps(S):
    """Two decoding steps in one recording (two plans: the buffers are back where they were), replayed with other
    inputs, beside the same steps eagerly on a cache of its own."""
    import torch
    from paper_2607_14557_amd.runner import PagedCache, record
    H, KV, D, B, rows = 8, 2, 128, 3, 4
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    normal = lambda n: torch.empty(rows, n * D, device="cuda").normal_(0, 1, generator=gen).bfloat16()
    cu = dev(np.array([0, 1, 2, 3]))
    caches = [PagedCache(H, KV, D, 1, 60, 16, B, 320, 300) for _ in range(2)]
    start = [normal(KV).repeat(40, 1)[:150] for _ in range(2)]
    cu0 = dev(np.array([0, 100, 101, 150]))
    for c in caches:
        c.store(0, start[0], start[1], 150, c.plan(cu0, 150))
        c.check()
    q, k, v = normal(H), normal(KV), normal(KV)
    outs = [[torch.zeros(rows, H * D, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in caches]
    st = torch.cuda.Stream()

    def two(c, out, stream):
        for i in range(2):
            c.store(0, k, v, rows, c.plan(cu, rows, stream=stream), stream=stream)
            c.attend(0, q, out[i], cu, rows, stream=stream)

    torch.cuda.synchronize()
    g = record(lambda: two(caches[0], outs[0], st), st)
    for i in range(5):
        for t, n in ((q, H), (k, KV), (v, KV)):
            t.copy_(normal(n))
        torch.cuda.synchronize()
        g.replay(st)
        st.synchronize()
        two(caches[1], outs[1], None)
        torch.cuda.synchronize()
        for a, b in zip(*outs):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), i
        assert host(caches[0].lens).tolist() == host(caches[1].lens).tolist() == [102 + 2 * i, 3 + 2 * i, 51 + 2 * i]
        assert torch.equal(caches[0].table, caches[1].table)
    g.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_beside_the_layer(S, dtype):
    """The K | V rows that a layer call leaves, stored in pages: attention of the call's own q rows over the pages is
    what the layer's attention left, to the roundings of both (its float64 value is held to in the layer's own tests)."""
    import torch
    from paper_2607_14557_amd.runner import PagedCache, SeerStack, dims_for
    from workloads.generate import round_to_dtype
    rng = np.random.default_rng(5)
    d, H, D, I = (512, 4, 128, 1024) if dtype == "bf16" else (256, 4, 64, 688)
    lens, rows = [100, 1, 213, 64], 512
    T, B = sum(lens), len(lens)
    W = {k: round_to_dtype(rng.standard_normal(s) * 0.04, dtype) for k, s in
         (("wq", (d, d)), ("wk", (d, d)), ("wv", (d, d)), ("wo", (d, d)), ("wg", (I, d)), ("wu", (I, d)), ("wd", (d, I)))}
    W.update(g1=np.ones(d), g2=np.ones(d))
    st = SeerStack(dims_for(d, H, D, I, dtype), 1, rows)
    st.set_layer(0, upload_weights(W, dtype))
    x = np.zeros((rows, d))
    x[:T] = rng.standard_normal((T, d))
    xd, cu = dev(x, dtype), dev(np.concatenate([[0], np.cumsum(lens)]))
    y = torch.zeros_like(xd)
    st.layer(0, xd, y, cu, None, B, rows)
    c = PagedCache(H, H, D, 1, 40, 16, B, 256, rows, dtype=dtype, v_f16=dtype == "bf16")
    c.store_layer(0, st, rows, c.plan(cu, rows))
    off = S.seer_layer_workspace_offsets(st.dims, rows)
    q = view_ws(st.workspace, off[0], rows, 3 * d, dtype)[:, :d]
    o = view_ws(st.workspace, off[1], rows, d, dtype)
    out = torch.zeros(rows, d, dtype=xd.dtype, device="cuda")
    c.attend(0, q, out, cu, rows, S.SEER_MASK_NONE)
    c.check()
    a, b = host(out)[:T], host(o)[:T]
    # both are within 2 u_p A + u_o |o| of the value (gqa_util), A of the order of |v|: the layer's v are about unit
    tol = 2 * (2 * 2.0 ** -11 + 2.0 ** -8) * max(1.0, float(np.abs(b).max())) if dtype == "bf16" else 2e-4
    diff = float(np.abs(a - b).max())
    log("%s: pages against the layer: %.3g (limit %.3g)" % (dtype, diff, tol))
    assert np.abs(b).max() > 0.1 and diff <= tol
    other = PagedCache(H, H, D, 1, 4, 16, B, 64, rows, dtype="f32" if dtype == "bf16" else "bf16")
    with pytest.raises(ValueError):
        other.store_layer(0, st, rows)
    with pytest.raises(ValueError):
        c.plan(cu, rows + 1)


def test_another_current_device(S, monkeypatch):
    """A cache's calls while another device is current are refused."""
    import torch
    p = Program(S, "bf16")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        p.c.plan(dev(np.zeros(6, int)), 8)
