"""The attention's workspace (no GPU): what a call needs never passes what was asked for with more rows or sequences."""
import ctypes
import os
import random

import pytest

FAKE = 1 << 20   # a non-null, aligned address that is never dereferenced


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    if not os.path.exists(seer.LIB_PATH):
        pytest.skip("libseer.so not built")
    seer.load_library()
    return seer


def test_never_less_for_more(S):
    rng = random.Random(2)
    for _ in range(4000):
        kv = rng.choice([1, 2, 4, 8, 32])
        heads, bf16 = kv * rng.choice([1, 2, 4, 7, 16, 71]), rng.random() < 0.7
        d = S.seer_attn_desc(heads, kv, rng.choice([64, 128]), S.SEER_DTYPE_BF16 if bf16 else S.SEER_DTYPE_F32, 0, 0.0)
        rows, batch = int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 11))
        less = rng.randint(1, rows), rng.randint(1, batch)
        most = S.seer_attn_workspace_bytes(d, rows, batch)
        for r, b in (less, (rows, less[1]), (less[0], batch), (rows, 1)):
            assert S.seer_attn_workspace_bytes(d, r, b) <= most, (heads, kv, rows, batch, r, b)


def test_fewer_sequences_than_were_asked_for(S):
    """64 rows, 32 heads on 8, in up to 64 sequences: a call with one sequence is not refused for its workspace."""
    d, pages = S.seer_attn_desc(32, 8, 128, S.SEER_DTYPE_BF16, 0, 0.0), S.seer_page_desc(64, 100, 10)
    n = S.seer_attn_workspace_bytes(d, 64, 64)
    # the next check after the workspace's is the pool's
    assert S.load_library().seer_attn_paged(ctypes.byref(d), ctypes.byref(pages), S.SEER_MASK_CAUSAL, FAKE, 4096, FAKE * 2, 4096,
                                            64, FAKE, None, 1, None, FAKE, FAKE, None, 0, FAKE, n, None) == S.SEER_EINVAL
    assert "required pointer" in S.seer_last_error()
