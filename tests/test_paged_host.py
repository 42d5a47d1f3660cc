"""Host-side checks of the paged entry points (no GPU): every refusal comes
back as its status code before anything is launched."""
import ctypes
import os

import pytest

FAKE = 1 << 20   # a non-null, aligned address that is never dereferenced


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    if not os.path.exists(seer.LIB_PATH):
        pytest.skip("libseer.so not built")
    seer.load_library()
    return seer


def heads(S, **kw):
    a = dict(h=8, kv=2, d=128, t=S.SEER_DTYPE_BF16, flags=0, scale=0.0)
    a.update(kw)
    return S.seer_attn_desc(a["h"], a["kv"], a["d"], a["t"], a["flags"], a["scale"])


def pages(S, size=64, n=100, width=10):
    return S.seer_page_desc(size, n, width)


def test_pool_bytes(S):
    assert S.seer_page_pool_bytes(heads(S), pages(S)) == 100 * 2 * 2 * 64 * 128 * 2
    f32 = heads(S, d=80, t=S.SEER_DTYPE_F32)
    assert S.seer_page_pool_bytes(f32, pages(S, size=16)) == 100 * 2 * 2 * 16 * 80 * 4
    # past 32 bits
    assert S.seer_page_pool_bytes(heads(S, kv=8), pages(S, n=1 << 20)) == (1 << 20) * 2 * 8 * 64 * 128 * 2
    for bad in (heads(S, h=7), heads(S, kv=0), heads(S, h=0), heads(S, d=96), heads(S, d=0), heads(S, t=9),
                heads(S, flags=2), heads(S, scale=float("nan")), heads(S, scale=float("inf")), heads(S, scale=-0.1),
                heads(S, t=S.SEER_DTYPE_F32, d=132), heads(S, t=S.SEER_DTYPE_F32, d=30),
                heads(S, t=S.SEER_DTYPE_F32, flags=S.SEER_ATTN_V_F16), heads(S, h=1 << 18, kv=1)):
        assert S.seer_page_pool_bytes(bad, pages(S)) == 0 and S.seer_last_error()
        assert S.seer_attn_workspace_bytes(bad, 10, 1) == 0
    for bad in (pages(S, size=8), pages(S, size=48), pages(S, size=512), pages(S, n=0), pages(S, width=0),
                pages(S, size=256, n=1 << 23)):
        assert S.seer_page_pool_bytes(heads(S), bad) == 0 and S.seer_last_error()


def test_plan_refusals(S):
    names = ("held", "keep", "cu", "used", "batch", "rows", "free", "free_in", "free_out", "table", "kv_len", "slots",
             "status")

    def call(desc=None, **kw):
        a = dict(held=FAKE, keep=FAKE + 4096, cu=FAKE, used=None, batch=2, rows=10, free=FAKE, free_in=FAKE,
                 free_out=FAKE + 256, table=FAKE, kv_len=FAKE + 8192, slots=FAKE, status=FAKE)
        a.update(kw)
        return S.load_library().seer_page_plan(ctypes.byref(desc or pages(S)), *[a[n] for n in names], None)

    for n in ("held", "keep", "cu", "free", "free_in", "free_out", "table", "kv_len", "slots", "status"):
        assert call(**{n: None}) == S.SEER_EINVAL, n
    assert call(batch=0) == S.SEER_EINVAL
    assert call(batch=4097) == S.SEER_EUNSUPPORTED
    assert call(rows=-1) == S.SEER_EINVAL
    assert call(free_out=FAKE) == S.SEER_EINVAL and "free_out" in S.seer_last_error()
    assert call(kv_len=FAKE) == S.SEER_EINVAL
    assert call(kv_len=FAKE + 4096) == S.SEER_EINVAL
    assert call(pages(S, size=24)) == S.SEER_EUNSUPPORTED
    assert S.load_library().seer_page_plan(None, *[FAKE] * 13, None) == S.SEER_EINVAL


def test_store_refusals(S):
    def call(d=None, pg=None, k=FAKE, ks=256, v=FAKE, vs=256, rows=4, slots=FAKE, pool=FAKE):
        return S.load_library().seer_kv_store(ctypes.byref(d or heads(S)), ctypes.byref(pg or pages(S)), k, ks, v, vs,
                                              rows, slots, pool, None)

    for kw in (dict(k=None), dict(v=None), dict(slots=None), dict(pool=None), dict(rows=0), dict(k=FAKE + 8),
               dict(v=FAKE + 2), dict(pool=FAKE + 4), dict(ks=255), dict(ks=248), dict(vs=260), dict(vs=-256),
               dict(ks=(1 << 24) + 8)):
        assert call(**kw) == S.SEER_EINVAL, kw
    assert call(d=heads(S, d=96)) == S.SEER_EUNSUPPORTED
    assert call(pg=pages(S, size=17)) == S.SEER_EUNSUPPORTED


def attn_args(S, d, kw):
    ws = S.seer_attn_workspace_bytes(d, kw.get("rows", 10), kw.get("batch", 2)) if kw.get("rows", 10) > 0 else 0
    a = dict(mask=S.SEER_MASK_CAUSAL, q=FAKE, qs=1024, k=FAKE * 2, ks=256, v=FAKE * 3, vs=256, out=FAKE * 4, os=1024,
             rows=10, cu=FAKE, used=None, batch=2, pool=FAKE * 5, table=FAKE, kv_len=FAKE, bits=None, words=0, ws=FAKE,
             ws_bytes=ws)
    a.update(kw)
    return a


def prompt(S, d=None, **kw):
    d = d or heads(S)
    a = attn_args(S, d, kw)
    return S.load_library().seer_attn_prompt(ctypes.byref(d), *[a[n] for n in (
        "mask", "q", "qs", "k", "ks", "v", "vs", "out", "os", "rows", "cu", "used", "batch", "ws", "ws_bytes")], None)


def paged(S, d=None, pg=None, **kw):
    d = d or heads(S)
    a = attn_args(S, d, kw)
    return S.load_library().seer_attn_paged(ctypes.byref(d), ctypes.byref(pg or pages(S)), *[a[n] for n in (
        "mask", "q", "qs", "out", "os", "rows", "cu", "used", "batch", "pool", "table", "kv_len", "bits", "words", "ws",
        "ws_bytes")], None)


def test_attention_refusals(S):
    for call in (prompt, paged):
        for kw in (dict(q=None), dict(out=None), dict(cu=None), dict(ws=None), dict(batch=0), dict(rows=0),
                   dict(rows=-5), dict(mask=3), dict(mask=-1), dict(q=FAKE + 2), dict(out=FAKE + 8), dict(qs=1020),
                   dict(qs=1016), dict(os=512), dict(os=1028), dict(out=FAKE), dict(ws=FAKE + 16)):
            assert call(S, **kw) == S.SEER_EINVAL, (call.__name__, kw)
        assert call(S, heads(S, d=80)) == S.SEER_EUNSUPPORTED
        assert call(S, heads(S, t=0)) == S.SEER_EUNSUPPORTED
        assert call(S, heads(S, h=9)) == S.SEER_EINVAL
        assert call(S, rows=1 << 28) == S.SEER_EUNSUPPORTED
        need = S.seer_attn_workspace_bytes(heads(S), 10, 2)
        assert need > 0 and call(S, ws_bytes=need - 1) == S.SEER_EWORKSPACE
        assert "workspace" in S.seer_last_error()
    for kw in (dict(k=None), dict(v=None), dict(ks=128), dict(vs=257), dict(k=FAKE + 4), dict(out=FAKE * 2),
               dict(out=FAKE * 3), dict(mask=S.SEER_MASK_TREE)):
        assert prompt(S, **kw) == S.SEER_EINVAL, kw
    for kw in (dict(pool=None), dict(table=None), dict(kv_len=None), dict(pool=FAKE + 8), dict(out=FAKE * 5),
               dict(mask=S.SEER_MASK_TREE), dict(mask=S.SEER_MASK_TREE, bits=FAKE, words=0)):
        assert paged(S, **kw) == S.SEER_EINVAL, kw
    assert paged(S, pg=pages(S, size=8)) == S.SEER_EUNSUPPORTED


def test_attention_of_more_workgroups_than_a_launch_has(S):
    """2^30 rows of one fp32 head are 2^26 workgroups of 16."""
    d = heads(S, h=1, kv=1, d=4, t=S.SEER_DTYPE_F32)
    n = S.seer_attn_workspace_bytes(d, 1 << 30, 1)
    assert n > 0
    assert S.load_library().seer_attn_prompt(ctypes.byref(d), S.SEER_MASK_CAUSAL, FAKE, 4, FAKE * 2, 4, FAKE * 3, 4,
                                             FAKE * 4, 4, 1 << 30, FAKE, None, 1, FAKE, n, None) == S.SEER_EUNSUPPORTED
    assert "workgroups" in S.seer_last_error()


def test_cache_refusals(S):
    """Rows and per-request arrays shorter than what the kernels read."""
    import torch
    from paper_2607_14557_amd.runner import PagedCache
    c = PagedCache(2, 1, 64, 1, 4, 16, 3, 32, 8, device="cpu")
    cu, three, x = torch.zeros(4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(8, 128, dtype=torch.bfloat16)
    k = x[:, :64]
    for call in (lambda: c.plan(cu, 9), lambda: c.plan(cu[:3], 8), lambda: c.plan(cu, 8, three[:2]),
                 lambda: c.plan(cu, 8, None, three[:1]), lambda: c.store(0, k, k, 9),
                 lambda: c.attend(0, x, x.clone(), cu[:3], 8), lambda: c.attend(0, x, x.clone(), cu, 9),
                 lambda: c.attend(0, x, x.clone(), cu, 8, seqused=three[:2]),
                 lambda: c.prompt(x, k, k, x.clone(), cu[:3], 8), lambda: c.prompt(x, k, k, x.clone(), cu, 9)):
        with pytest.raises(ValueError):
            call()
