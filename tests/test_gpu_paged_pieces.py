"""Cut lines of the attention with grouped heads in which workgroups take several pieces, one after the other, and calls
with more requests than a workgroup has threads: against the oracle, with values that show a lost or doubled block.
The form of each launch is asked from the rule itself (dispatch.h, compiled for the host)."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from gqa_blocks import block_values, check_blocks, u_p
from gqa_util import TYPES, U
from oracle.paged import sees
from test_dispatch import CXX, _ask
from test_dispatch_gqa import RULE
from test_gpu_attn_gqa import Paged, Prompt, S, _tree      # noqa: F401 (S: the fixture)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(CXX is None, reason="no host C++ compiler")]

FORM = RULE + """
int answer(const long long* v) {
  const GqaLaunch g = launch(v);
  const GqaRule r = gqa_rule(g);
  const int tiles = (int)gqa_tiles(g, r.rt);
  return (r.rt / 16 * 10000 + r.grid) * 4 + r.cut * 2 + (tiles <= r.grid / 2);
}
"""


class Blocks(Paged):
    """A Paged call whose keys are small and whose values are those of block_values."""

    def __init__(self, S, kind, H, KV, D, past, new, seed=1, **kw):
        super().__init__(S, kind, H, KV, D, past, new, seed=seed, factor=0.3, **kw)
        import torch
        v = np.concatenate([block_values(n, KV, D) for n in self.kv]).reshape(-1, KV * D)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed + 100)
        k = torch.empty(v.shape, device="cuda").normal_(0.0, 1.0, generator=gen).to(self.qt)
        vd = torch.from_numpy(v).to(self.vt).cuda()
        S.seer_kv_store(self.desc, self.pages, k, KV * D, vd, KV * D, len(v), dev(self.slots), self.pool)
        self.kh, self.vh = host(k).reshape(-1, KV, D), v.reshape(-1, KV, D)

    def form(self, tmp_path):
        """(rows of a tile, cut, workgroups, few enough tiles for runs) of the launch."""
        H, KV, D = self.shape
        f = _ask(tmp_path, FORM, [(H, KV, D, self.rows, len(self.new), self.W * self.page, 0, int(self.kind != "f32"))])[0]
        return f // 4 // 10000 * 16, bool(f & 2), f // 4 % 10000, bool(f & 1)

    def line(self, rt):
        """Blocks of the line of this call's own lengths."""
        H, KV, _ = self.shape
        return KV * sum(-(-n * (H // KV) // rt) * max(1, -(-k // 64)) for n, k in zip(self.new, self.kv))

    def check_blocks(self, mask, fine):
        H, KV, D = self.shape
        got, q = host(self.out), host(self.q).reshape(-1, H, D)
        assert (got[self.T:] == 9.0).all(), "rows behind the last sequence are left as they were"
        got, worst, at = got.reshape(-1, H, D), 0.0, 0
        q_type, v_type = TYPES[self.kind]
        for b, (s, n, L) in enumerate(zip(self.cu, self.new, self.kv)):
            if n:
                seen = sees(mask, n, L, None if self.bits is None else self.bits[s:s + n])
                worst = max(worst, check_blocks(got[s:s + n], q[s:s + n], self.kh[at:at + L], self.vh[at:at + L], seen,
                                                u_p(v_type, fine), U[q_type], "request %d of %d keys" % (b, L)))
            at += L
        return worst


def _run(tmp_path, p, mask, rt, runs, what):
    got = p.form(tmp_path)
    assert got[:2] == (rt, True), (what, got)
    assert got[3] == runs and (runs or p.line(rt) > got[2]), (what, got, p.line(rt))
    log("%s: %d blocks over %d workgroups%s" % (what, p.line(rt), got[2], ", in runs" if runs else ""))
    p.run(mask)
    log("  %.3g of the bound" % p.check_blocks(mask, rt == 32 and p.kind == "bf16"))
    first = host(p.out).tobytes()
    p.out.fill_(9.0)
    p.run(mask)
    assert host(p.out).tobytes() == first, "the same call twice gives other bits"


@pytest.mark.parametrize("kind,H,KV,D,B", [("bf16", 28, 4, 128, 64), ("v16", 28, 4, 128, 64), ("bf16", 14, 2, 64, 256),
                                           ("f32", 8, 8, 64, 64)])
def test_equal_stretches_over_ragged_tokens(S, tmp_path, kind, H, KV, D, B):
    """Single tokens over 0 to 4000 keys: stretches that end one tile, hold whole ones and open another."""
    rng = np.random.default_rng(5)
    past = [int(4000 ** rng.random()) for _ in range(B)]
    past[3], past[10], past[40], past[B - 1] = 0, 4000, 3999, 64
    if kind == "f32":
        past = [n // 2 for n in past]
    p = Blocks(S, kind, H, KV, D, past, [1] * B, page=64, width=250 if B > 128 else 63)
    _run(tmp_path, p, "causal", 16 if kind == "f32" else 32, False, "%s %d/%d of %d" % (kind, H, KV, D))


@pytest.mark.parametrize("kind,H,KV,D,B,new", [("bf16", 16, 1, 128, 200, 1), ("v16", 16, 1, 128, 200, 1),
                                               ("bf16", 8, 1, 64, 300, 5), ("f32", 4, 1, 64, 300, 1)])
def test_more_requests_than_threads(S, tmp_path, kind, H, KV, D, B, new):
    """Every place in use, equal stretches: a thread has two or three requests."""
    rng = np.random.default_rng(B)
    past = [int(1500 ** rng.random()) for _ in range(B)]
    past[0], past[1], past[B - 1], past[B // 2] = 0, 3900, 2600, 64
    lens = [new if new == 1 else int(rng.integers(0, 2 * new)) for _ in range(B)]
    p = Blocks(S, kind, H, KV, D, past, lens, page=64, width=260 if new > 1 else 63)
    _run(tmp_path, p, "causal", 16 if kind == "f32" else 32, False, "%s %d requests" % (kind, B))


@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 8, 2, 128), ("v16", 14, 2, 64), ("f32", 8, 2, 128)])
@pytest.mark.parametrize("B", [300, 700])
def test_few_rows_in_a_cache_of_many_places(S, tmp_path, kind, H, KV, D, B):
    """Four rows in B places, keys in runs."""
    past, new = [0] * B, [0] * B
    for b, n in ((2, 7900), (B // 2, 1), (B // 2 + 1, 2049), (B - 1, 640)):
        past[b], new[b] = n, 1
    past[5] = 333                                      # in the cache, without a row in this call
    p = Blocks(S, kind, H, KV, D, past, new, page=64, width=125, pad=2)
    _run(tmp_path, p, "causal", 16 if kind == "f32" else 32, True, "%s %d places" % (kind, B))


@pytest.mark.parametrize("kind,mask", [("bf16", "tree"), ("v16", "causal")])
def test_tiles_of_128_rows_over_many_requests(S, tmp_path, kind, mask):
    """300 requests of a few rows with 16 heads on one: 128-row tiles, cut, two requests a thread."""
    rng = np.random.default_rng(8)
    B = 300
    new = [int(rng.integers(0, 9)) for _ in range(B)]
    past = [int(900 ** rng.random()) for _ in range(B)]
    past[7], past[200] = 3500, 0
    bits = sum([_tree(rng, n) for n in new], []) if mask == "tree" else None
    p = Blocks(S, kind, 16, 1, 128, past, new, page=16, width=250, bits=bits, words=1 if bits else 0)
    _run(tmp_path, p, mask, 128, False, "%s %s" % (kind, mask))


@pytest.mark.parametrize("kind,H,KV,D,past,new", [("bf16", 40, 1, 128, 32770, 1), ("v16", 14, 2, 64, 20000, 3),
                                                  ("f32", 8, 2, 64, 16384, 2), ("bf16", 16, 2, 128, 12003, 60)])
def test_long_contexts(S, tmp_path, kind, H, KV, D, past, new):
    """One request of many blocks, and one of a few keys beside it."""
    p = Blocks(S, kind, H, KV, D, [past, 5], [new, 1], page=256)
    rt, cut, grid, _ = p.form(tmp_path)
    assert cut
    p.run("causal")
    log("%s %d keys, %d rows, tiles of %d: %.3g of the bound" %
        (kind, past, new, rt, p.check_blocks("causal", rt == 32 and kind == "bf16")))


@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 8, 2, 128), ("v16", 2, 2, 64), ("f32", 4, 1, 64)])
def test_uncut_walks(S, kind, H, KV, D):
    """A prompt's tiles, each one walk over all keys."""
    import torch
    lens = [700, 65, 1300] if kind != "f32" else [300, 65]
    p = Prompt(S, kind, H, KV, D, lens, factor=0.3)
    v = np.concatenate([block_values(n, KV, D) for n in lens]).reshape(-1, KV * D)
    p.v[:p.T] = torch.from_numpy(v).to(p.vt).cuda()
    p.run(S.SEER_MASK_CAUSAL)
    got, q, k = host(p.out)[:, :H * D].reshape(-1, H, D), host(p.q).reshape(-1, H, D), host(p.k).reshape(-1, KV, D)
    for s, n in zip(p.cu, lens):
        at = [i for i in range(n) if i < 3 or i % 64 in (0, 63) or i == n - 1]
        for i in at:
            check_blocks(got[s + i:s + i + 1], q[s + i:s + i + 1], k[s:s + i + 1], v[s:s + i + 1].reshape(-1, KV, D),
                         np.ones((1, i + 1), bool), u_p(TYPES[kind][1], False), U[TYPES[kind][0]], "row %d of %d" % (i, n))
