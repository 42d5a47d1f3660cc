"""Large finite values: the sums of the attention with grouped heads stay finite where the header says so."""
import numpy as np
import pytest

from gpu_util import dev, host, log
from gqa_util import TYPES
from test_gpu_attn_gqa import Paged, Prompt, S      # noqa: F401 (S: the fixture)

pytestmark = pytest.mark.gpu


def _fill(p, scores, values):
    """Keys of request 0 whose scores against p's (equal) query rows and heads are `scores`, every value of key t values[t]."""
    import torch
    H, KV, D = p.shape
    p.q.copy_(p.q[:1, :D].repeat(p.q.shape[0], H))
    q = p.q[0, :D].float()
    k = (q[None, :] * (torch.as_tensor(scores, dtype=torch.float32, device="cuda") * D ** 0.5 / q.square().sum())[:, None]).to(p.qt)
    v = torch.as_tensor(values, dtype=torch.float64, device="cuda")[:, None].expand(-1, D).to(p.vt).contiguous()
    p.S.seer_kv_store(p.desc, p.pages, k, D, v, D, len(scores), dev(p.slots), p.pool)


@pytest.mark.parametrize("H,new", [(1, 1), (1, 40), (8, 300)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_a_large_value_behind_the_first_keys(S, kind, H, new):
    """A key with 22,026 times the weight of those before it, and a value near the type's end."""
    n = 1000
    p = Paged(S, kind, H, 1, 64, [n - new], [new])
    scores, values = np.zeros(n), np.ones(n)
    scores[400], values[400] = 10.0, 60000.0 if kind == "v16" else 1e36
    _fill(p, scores, values)
    p.run("none")
    log("%s %d rows: %.3g of the bound" % (kind, new, p.check("none", rows=[0, new // 2, new - 1])))


@pytest.mark.parametrize("H,new", [(1, 1), (1, 40), (8, 300)])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_all_values_as_large_as_the_header_allows(S, kind, H, new):
    """2^126 / (keys + 64), with scores that rise by 3 a tile over the first eight."""
    n = 1000
    p = Paged(S, kind, H, 1, 64, [n - new], [new])
    rng = np.random.default_rng(6)
    scores = rng.uniform(-1, 1, n) + np.minimum(np.arange(n) // 64, 8) * 3.0
    _fill(p, scores, np.full(n, 2.0 ** 126 / (n + 64) * 0.99))
    p.run("none")
    assert np.isfinite(host(p.out)[:p.T]).all()
    log("%s %d rows: %.3g of the bound" % (kind, new, p.check("none", rows=[0, new // 2, new - 1])))


@pytest.mark.parametrize("kind", list(TYPES))
def test_a_large_value_in_a_prompt(S, kind):
    """The same in tiles of 128 rows, each one walk over all its keys."""
    H, KV, D = (32, 8, 128) if kind != "f32" else (4, 1, 64)
    lens = [1300, 600, 600, 600, 900] if kind != "f32" else [450, 600]
    p = Prompt(S, kind, H, KV, D, lens)
    p.q.copy_(p.q[:1, :D].repeat(p.rows, H))
    one = (p.q[0, :D].float() * (10.0 * D ** 0.5 / p.q[0, :D].float().square().sum())).to(p.qt).repeat(KV)
    p.k.zero_()
    p.v.fill_(1.0)
    for s in p.cu[:-1]:
        p.k[s + 400], p.v[s + 400] = one, 60000.0 if kind == "v16" else 1e36
    p.run(S.SEER_MASK_CAUSAL)
    log("%s: %.3g of the bound" % (kind, p.check("causal", rows=[0, 127, 399, 400, 449, 599, 1299])))
