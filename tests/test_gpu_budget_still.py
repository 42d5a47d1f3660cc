"""Keys that are stored as they are (BudgetCache without a rotation, rows of a layer): bit for bit, whatever the bits."""
import numpy as np
import pytest

from gpu_util import dev
from gqa_util import torch_types

pytestmark = pytest.mark.gpu
ROWS, B = 70, 2


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    seer.load_library()
    return seer


def _any_bits(t, n, width, seed):
    """Rows of arbitrary bits, with -0 beside finite values and infinities."""
    import torch
    word = {2: (torch.int16, np.int16), 4: (torch.int32, np.int32)}[torch.empty(0, dtype=t).element_size()]
    r = np.random.default_rng(seed)
    lo, hi = np.iinfo(word[1]).min, np.iinfo(word[1]).max
    x = torch.from_numpy(r.integers(lo, hi, (n, width), endpoint=True, dtype=word[1])).cuda().view(t)
    x[0, 0], x[0, 1], x[1, 0], x[1, 1], x[2, 0], x[2, 1] = float("inf"), 1.5, 2.0, float("-inf"), -0.0, -0.0
    return x


def _bits(x):
    import torch
    return x.view(torch.int16 if x.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("kind,H,KV,D", [("bf16", 4, 2, 128), ("v16", 6, 2, 64), ("f32", 3, 3, 80), ("f32", 2, 1, 4)])
def test_as_a_cache_without_positions(S, kind, H, KV, D):
    import torch
    from paper_2607_14557_amd.runner import BudgetCache, PagedCache
    qt, vt = torch_types(kind)
    args = dict(dtype="f32" if kind == "f32" else "bf16", v_f16=kind == "v16")
    a, b = PagedCache(H, KV, D, 1, 10, 16, B, 80, ROWS, **args), BudgetCache(H, KV, D, 1, 10, 16, B, 80, ROWS, **args)
    q, k, v = _any_bits(qt, ROWS, H * D, 1), _any_bits(qt, ROWS, KV * D, 2), _any_bits(vt, ROWS, KV * D, 3)
    cu = dev(np.array([0, 40, 61]))
    for c in (a, b):
        c.plan(cu, ROWS)
    out, q0 = torch.zeros_like(q), q.clone()
    a.store(0, k, v, ROWS)
    b.store(0, k, v, ROWS, q=q, q_out=out)
    assert torch.equal(_bits(a.pools[0]), _bits(b.pools[0]))
    assert torch.equal(_bits(out)[:61], _bits(q)[:61]) and (_bits(out)[61:] == 0).all() and torch.equal(_bits(q), _bits(q0))
    b.store(0, k, v, ROWS, q=q)                          # in place
    assert torch.equal(_bits(q), _bits(q0)) and torch.equal(_bits(a.pools[0]), _bits(b.pools[0]))
    ko, k0 = torch.zeros_like(k), k.clone()
    for inverse in (False, True):
        b.rotate(q, k, ROWS, q_out=out.zero_(), k_out=ko.zero_(), inverse=inverse)
        assert torch.equal(_bits(out)[:61], _bits(q)[:61]) and torch.equal(_bits(ko)[:61], _bits(k)[:61])
        assert (_bits(out)[61:] == 0).all() and (_bits(ko)[61:] == 0).all()
        b.rotate(q, k, ROWS, inverse=inverse)
        assert torch.equal(_bits(q), _bits(q0)) and torch.equal(_bits(k), _bits(k0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_layer(S, dtype):
    import torch
    from paper_2607_14557_amd.runner import BudgetCache, PagedCache, SeerStack, dims_for
    d, H, D, I = 256, 2, 128, 512
    stack = SeerStack(dims_for(d, H, D, I, dtype), 1, ROWS)
    es = 2 if dtype == "bf16" else 4
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    at = S.seer_layer_workspace_offsets(stack.dims, ROWS)[0]
    stack.workspace[at:at + ROWS * 3 * d * es].copy_(_any_bits(t, ROWS, 3 * d, 5).contiguous().view(torch.uint8).reshape(-1))
    cu = dev(np.array([0, 40, 61]))
    pools = []
    for cls in (PagedCache, BudgetCache):
        c = cls(H, H, D, 1, 10, 16, B, 80, ROWS, dtype=dtype, v_f16=dtype == "bf16")
        c.plan(cu, ROWS)
        c.store_layer(0, stack, ROWS)
        pools.append(c.pools[0])
    assert torch.equal(_bits(pools[0]), _bits(pools[1]))
