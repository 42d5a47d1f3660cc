"""The values of gqa_blocks on the CPU: a result with a block or a seam's key lost or doubled is refused, one that is
rounded as the kernels round is taken."""
import numpy as np
import pytest

from gqa_blocks import block_values, check_blocks, u_p
from gqa_util import TYPES, U
from oracle.paged import attend


def _bf16(x):
    import torch
    return torch.from_numpy(np.asarray(x, np.float64)).bfloat16().double().numpy()


def _weights(q, k, times):
    """float64 softmax attention of one head with key t counted times[t] times."""
    s = k @ q / np.sqrt(q.size)
    p = np.exp(s - s.max()) * times
    return p / p.sum()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,D", [(32771, 128), (12003, 128), (20001, 64), (700, 64), (130, 128)])
def test_lost_and_doubled_keys_are_found(kind, n, D):
    rng = np.random.default_rng(n)
    q, k = 0.2 * rng.standard_normal((1, 1, D)), rng.standard_normal((n, 1, D))
    v, seen = block_values(n, 1, D), np.ones((1, n), bool)
    v_type, fine = TYPES[kind][1], kind == "bf16"
    up, uo = u_p(v_type, fine), U[TYPES[kind][0]]
    rounded = (lambda x: _bf16(x)) if kind != "f32" else (lambda x: x.astype(np.float32).astype(float))

    def result(times):
        return rounded((_weights(q[0, 0], k[:, 0], times) @ v[:, 0])[None, None])

    assert check_blocks(result(np.ones(n)), q, k, v, seen, up, uo, "as it is") <= 1.0
    blocks = -(-n // 64)
    for b in sorted({0, 1, blocks // 3, blocks - 1}):
        lo, hi = 64 * b, min(64 * b + 64, n)
        for what, at in (("block", slice(lo, hi)), ("first key", slice(lo, lo + 1)), ("last key", slice(hi - 1, hi))):
            if what == "last key" and hi - lo < 64:
                continue                                 # the last block's end holds a 1
            for count in (0.0, 2.0):
                times = np.ones(n)
                times[at] = count
                with pytest.raises(AssertionError):
                    check_blocks(result(times), q, k, v, seen, up, uo, "%s of block %d times %g" % (what, b, count))


def test_a_lost_second_part_is_found():
    """Probabilities cut to their upper bf16 halves, their sum over the whole ones: 0.28% too little, more than the
    result's rounding alone in some dims."""
    n, D = 8000, 128
    rng = np.random.default_rng(3)
    q, k, v, seen = 0.2 * rng.standard_normal((1, 1, D)), rng.standard_normal((n, 1, D)), block_values(n, 1, D), np.ones((1, n), bool)
    s = k[:, 0] @ q[0, 0] / np.sqrt(D)
    p = np.exp(s - s[:64].max())
    cut = (p.astype(np.float32).view(np.uint32) & 0xffff0000).view(np.float32).astype(float)
    one = _bf16((cut @ v[:, 0] / p.sum())[None, None])
    with pytest.raises(AssertionError):
        check_blocks(one, q, k, v, seen, u_p("bf16", True), U["bf16"], "one part")
    check_blocks(one, q, k, v, seen, u_p("bf16", False), U["bf16"], "one rounding more")
