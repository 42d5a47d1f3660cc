"""Host-side checks of a cache within a budget (no GPU): frequencies, and every refusal before anything is launched."""
import ctypes
import os
import types

import numpy as np
import pytest
import torch

from oracle.budget import frequencies

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


def rope(S, **kw):
    a = dict(layout=0, rot=0, scaling=0, original=2048, theta=10000.0, factor=4.0, low=1.0, high=4.0, magnitude=0.0)
    a.update(kw)
    return S.seer_rope_desc(*[a[n] for n in ("layout", "rot", "scaling", "original", "theta", "factor", "low", "high",
                                             "magnitude")])


@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "bands", "ramp"])
@pytest.mark.parametrize("rot", [0, 2, 10, 64, 112])
def test_turns(S, scaling, rot):
    kind = ["plain", "linear", "base", "bands", "ramp"].index(scaling)
    high = 32.0 if scaling == "ramp" else 4.0
    got = np.array(S.seer_rope_turns(rope(S, rot=rot, scaling=kind, factor=8.0, high=high, theta=500000.0), 128))
    want = frequencies(rot or 128, 500000.0, scaling, 8.0, 1.0, high, 2048) / (2 * np.pi)
    assert got.shape == want.shape and np.allclose(got, want, rtol=1e-13, atol=0)      # a few powers and products in fp64


def test_turns_refusals(S):
    bad = [dict(layout=2), dict(layout=-1), dict(rot=-2), dict(rot=3), dict(rot=130), dict(scaling=5), dict(scaling=-1),
           dict(theta=1.0), dict(theta=float("inf")), dict(theta=float("nan")), dict(scaling=1, factor=0.0),
           dict(scaling=2, factor=float("nan")), dict(scaling=3, low=0.0), dict(scaling=3, low=4.0), dict(scaling=4, high=0.5),
           dict(scaling=4, original=0), dict(scaling=3, high=float("inf")), dict(magnitude=-1.0),
           dict(magnitude=float("nan"))]
    for kw in bad:
        with pytest.raises(S.SeerError) as e:
            S.seer_rope_turns(rope(S, **kw), 128)
        assert e.value.code == S.SEER_EINVAL, kw
    for dim in (0, 1, 130):
        with pytest.raises(S.SeerError):
            S.seer_rope_turns(rope(S), dim)
    with pytest.raises(S.SeerError):
        S.seer_rope_turns(rope(S), 65)                     # the whole of an odd head
    assert len(S.seer_rope_turns(rope(S, rot=64), 65)) == 32
    assert S.load_library().seer_rope_turns(None, 128, (ctypes.c_double * 64)()) == S.SEER_EINVAL
    assert S.load_library().seer_rope_turns(ctypes.byref(rope(S)), 128, None) == S.SEER_EINVAL


def test_rope_rows_refusals(S):
    names = ("turns", "flags", "q", "qs", "k", "ks", "qo", "qos", "ko", "kos", "rows", "pos")

    def call(d=None, r=None, **kw):
        a = dict(turns=FAKE, flags=0, q=FAKE, qs=1536, k=2 * FAKE, ks=1536, qo=3 * FAKE, qos=1024, ko=4 * FAKE, kos=256, rows=4,
                 pos=FAKE)
        a.update(kw)
        return S.load_library().seer_rope_rows(ctypes.byref(d or heads(S)), ctypes.byref(r or rope(S)),
                                               *[a[n] for n in names], None)

    for n in ("turns", "q", "k", "qo", "ko", "pos"):
        assert call(**{n: None}) == S.SEER_EINVAL, n
    assert call(q=None, qo=None, k=None, ko=None) == S.SEER_EINVAL
    assert call(flags=2) == S.SEER_EINVAL and call(rows=0) == S.SEER_EINVAL
    for kw in (dict(qs=1020), dict(qs=1001), dict(ks=248), dict(qos=1016), dict(kos=255), dict(q=FAKE + 2), dict(ko=FAKE + 8),
               dict(qs=(1 << 24) + 8), dict(qo=FAKE), dict(ko=2 * FAKE), dict(qo=2 * FAKE), dict(ko=FAKE), dict(ko=3 * FAKE)):
        assert call(**kw) == S.SEER_EINVAL, kw
    assert call(d=heads(S, d=96)) == S.SEER_EUNSUPPORTED
    assert call(r=rope(S, layout=7)) == S.SEER_EINVAL
    assert call(d=heads(S, d=64), r=rope(S, rot=66)) == S.SEER_EINVAL


def test_store_refusals(S):
    names = ("turns", "q", "qs", "qo", "qos", "k", "ks", "v", "vs", "rows", "pos", "slots", "pool", "weight", "number")

    def call(d=None, p=None, r=None, **kw):
        a = dict(turns=FAKE, q=FAKE, qs=1024, qo=3 * FAKE, qos=1024, k=2 * FAKE, ks=256, v=FAKE, vs=256, rows=4, pos=FAKE,
                 slots=FAKE, pool=5 * FAKE, weight=FAKE, number=FAKE)
        a.update(kw)
        return S.load_library().seer_kv_store_rope(ctypes.byref(d or heads(S)), ctypes.byref(p or pages(S)),
                                                   ctypes.byref(r or rope(S)), *[a[n] for n in names], None)

    for n in ("turns", "q", "qo", "k", "v", "pos", "slots", "pool", "weight", "number"):
        assert call(**{n: None}) == S.SEER_EINVAL, n
    for kw in (dict(rows=0), dict(ks=248), dict(vs=8), dict(vs=257), dict(pool=FAKE + 8), dict(v=FAKE + 4),
               dict(qo=2 * FAKE), dict(qo=5 * FAKE), dict(qo=FAKE, v=3 * FAKE, q=3 * FAKE, k=FAKE)):
        assert call(**kw) == S.SEER_EINVAL, kw
    assert call(p=pages(S, size=24)) == S.SEER_EUNSUPPORTED and call(p=pages(S, n=0)) == S.SEER_EINVAL
    assert call(d=heads(S, h=7)) == S.SEER_EINVAL


def test_row_positions_refusals(S):
    def call(cu=FAKE, used=None, batch=2, seen=FAKE, base=None, status=None, rows=4, pos=FAKE, next=2 * FAKE):
        return S.load_library().seer_row_positions(cu, used, batch, seen, base, status, rows, pos, next, None)

    assert call(cu=None) == S.SEER_EINVAL and call(pos=None) == S.SEER_EINVAL
    assert call(batch=0) == S.SEER_EINVAL and call(rows=-1) == S.SEER_EINVAL
    assert call(next=FAKE) == S.SEER_EINVAL and call(base=2 * FAKE) == S.SEER_EINVAL
    assert call(rows=0, pos=None, next=None) == S.SEER_OK


def test_weights_refusals(S):
    names = ("mask", "q", "qs", "rows", "cu", "used", "batch", "last", "pool", "table", "kv", "bits", "words", "decay", "prev",
             "weight", "ws", "bytes")

    def call(d=None, p=None, **kw):
        d, p = d or heads(S), p or pages(S)
        a = dict(mask=1, q=FAKE, qs=1024, rows=4, cu=FAKE, used=None, batch=2, last=0, pool=FAKE, table=FAKE, kv=FAKE,
                 bits=None, words=0, decay=1.0, prev=FAKE, weight=FAKE, ws=FAKE, bytes=1 << 40)
        a.update(kw)
        a["decay"] = ctypes.c_float(a["decay"])
        return S.load_library().seer_attn_weights(ctypes.byref(d), ctypes.byref(p), *[a[n] for n in names], None)

    for n in ("q", "cu", "pool", "table", "kv", "weight", "ws"):
        assert call(**{n: None}) == S.SEER_EINVAL, n
    for kw in (dict(mask=3), dict(mask=-1), dict(mask=2), dict(mask=2, bits=FAKE), dict(rows=0), dict(batch=0), dict(last=-1),
               dict(decay=-0.5), dict(decay=float("nan")), dict(decay=float("inf")), dict(qs=1016), dict(qs=1023),
               dict(q=FAKE + 2), dict(pool=FAKE + 8), dict(ws=FAKE + 16)):
        assert call(**kw) == S.SEER_EINVAL, kw
    assert call(batch=4097) == S.SEER_EUNSUPPORTED
    assert call(rows=1 << 28) == S.SEER_EUNSUPPORTED
    assert call(batch=4096, p=pages(S, width=1 << 17)) == S.SEER_EUNSUPPORTED
    need = S.seer_attn_weights_workspace_bytes(heads(S), pages(S), 4, 2)
    assert need > 0 and call(bytes=need - 1) == S.SEER_EWORKSPACE
    for bad in ((heads(S, d=96), pages(S), 4, 2), (heads(S), pages(S, n=0), 4, 2), (heads(S), pages(S), 0, 2),
                (heads(S), pages(S), 4, 0), (heads(S), pages(S), 1 << 28, 2)):
        assert S.seer_attn_weights_workspace_bytes(*bad) == 0 and S.seer_last_error()


def test_evict_refusals(S):
    names = ("flags", "kv", "budget", "seen", "batch", "first", "recent", "table", "pool", "weight", "number", "wo", "no",
             "kept", "ws", "bytes")

    def call(d=None, p=None, **kw):
        a = dict(flags=0, kv=FAKE, budget=2 * FAKE, seen=3 * FAKE, batch=2, first=0, recent=0, table=FAKE, pool=FAKE,
                 weight=FAKE, number=2 * FAKE, wo=FAKE, no=2 * FAKE, kept=4 * FAKE, ws=FAKE, bytes=1 << 40)
        a.update(kw)
        return S.load_library().seer_kv_evict(ctypes.byref(d or heads(S)), ctypes.byref(p or pages(S)),
                                              *[a[n] for n in names], None)

    for n in ("kv", "budget", "seen", "table", "pool", "weight", "number", "wo", "no", "kept", "ws"):
        assert call(**{n: None}) == S.SEER_EINVAL, n
    for kw in (dict(flags=2), dict(batch=0), dict(first=-1), dict(recent=-1), dict(wo=8 * FAKE), dict(no=8 * FAKE),
               dict(kept=FAKE), dict(kept=3 * FAKE), dict(pool=FAKE + 8), dict(ws=FAKE + 16)):
        assert call(**kw) == S.SEER_EINVAL, kw
    assert call(batch=1 << 19) == S.SEER_EUNSUPPORTED
    need = S.seer_kv_evict_workspace_bytes(heads(S), pages(S), 2)
    assert need > 0 and call(bytes=need - 1) == S.SEER_EWORKSPACE
    assert S.seer_kv_evict_workspace_bytes(heads(S), pages(S), 0) == 0
    assert S.seer_kv_evict_workspace_bytes(heads(S, h=7), pages(S), 2) == 0


# ---- BudgetCache -----------------------------------------------------------------
H, KV, D, B, ROWS = 4, 2, 64, 3, 8
CALLS = ("seer_page_plan_latched", "seer_attn_paged", "seer_rope_rows", "seer_kv_store_rope", "seer_row_positions",
         "seer_attn_weights", "seer_kv_evict")


@pytest.fixture
def calls(S, monkeypatch):
    """The entry points' names as they are called, with no launch behind them."""
    from paper_2607_14557_amd import runner
    made = []
    for name in CALLS:
        monkeypatch.setattr(runner.S, name, lambda *a, _name=name, **kw: made.append((_name, a)))
    return made


def _cache(S, layers=2, **kw):
    from paper_2607_14557_amd.runner import BudgetCache
    return BudgetCache(H, KV, D, layers, 4, 16, B, 32, ROWS, rope=rope(S), device="cpu", **kw)


def _i32(n):
    return torch.zeros(n, dtype=torch.int32)


def _bf16(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def _refused(calls, call, match):
    before = len(calls)
    with pytest.raises(ValueError, match=match):
        call()
    assert len(calls) == before


def test_cache_takes(S, calls):
    c, cu = _cache(S), _i32(B + 1)
    q, k = _bf16(ROWS, H * D), _bf16(ROWS, KV * D)
    _refused(calls, lambda: c.store(0, k, k, ROWS), "last plan")
    _refused(calls, lambda: c.rotate(q, k, ROWS), "last plan")
    _refused(calls, lambda: c.plan(cu, ROWS, base=_i32(B).long()), "base")
    _refused(calls, lambda: c.plan(cu, ROWS, base=c._seen[1]), "base")
    c.plan(cu, ROWS, base=c.seen)
    _refused(calls, lambda: c.store(0, k.float(), k, ROWS), "k has")
    _refused(calls, lambda: c.store(0, k, k.half(), ROWS), "v has")
    _refused(calls, lambda: c.store(0, k, k, ROWS, q=q[:, ::2]), "q has")
    _refused(calls, lambda: c.store(0, k, k, ROWS, q=q, q_out=k), "q_out has")
    _refused(calls, lambda: c.store(0, k, k, ROWS, positions=_i32(ROWS - 1)), "positions")
    _refused(calls, lambda: c.rotate(q, q[:, :KV * D - 1], ROWS), "k has")
    _refused(calls, lambda: c.rotate(q[:3], k, ROWS), "q has")
    _refused(calls, lambda: c.weigh(0, k, cu, ROWS), "q has")
    _refused(calls, lambda: c.weigh(0, q, cu.long(), ROWS), "cu")
    _refused(calls, lambda: c.weigh(0, q, cu, ROWS + 1), "max_rows")
    _refused(calls, lambda: c.weigh(0, q, cu, ROWS, tree_bits=_i32(ROWS)), "tree_bits")
    _refused(calls, lambda: c.evict(0, _i32(B - 1)), "budget")
    c.store(0, k, k, ROWS, q=q)
    c.rotate(q, None, ROWS)
    c.weigh(0, q, cu, ROWS)
    assert [n for n, _ in calls] == ["seer_page_plan_latched", "seer_row_positions", "seer_kv_store_rope", "seer_rope_rows",
                                     "seer_attn_weights"]
    assert calls[3][1][6] is None and calls[3][1][10] is None              # no k


def test_cut_layers(S, calls):
    """A cut layer takes no call before the plan; the plan keeps what the cut kept, and refuses a cut of some layers."""
    c, cu, budget = _cache(S), _i32(B + 1), _i32(B)
    q, k = _bf16(ROWS, H * D), _bf16(ROWS, KV * D)
    c.plan(cu, ROWS)
    c.evict(0, budget)
    for call in (lambda: c.store(0, k, k, ROWS), lambda: c.attend(0, q, q.clone(), cu, ROWS), lambda: c.weigh(0, q, cu, ROWS),
                 lambda: c.evict(0, budget)):
        _refused(calls, call, "is cut")
    c.attend(1, q, q.clone(), cu, ROWS)
    _refused(calls, lambda: c.plan(cu, ROWS), "1 of 2 layers")
    c.evict(1, budget)
    c.plan(cu, ROWS)
    assert calls[-2][0] == "seer_page_plan_latched" and calls[-2][1][2] is c.kept
    c.store(0, k, k, ROWS)
    c.evict(0, budget)
    c.evict(1, budget)
    keep = _i32(B)
    c.plan(cu, ROWS, keep)
    assert calls[-2][1][2] is keep
    c.refused.fill_(S.SEER_PAGES_EXHAUSTED)                               # the plan was refused: the cut still stands
    with pytest.raises(S.SeerError):
        c.check(types.SimpleNamespace(synchronize=lambda: None))
    _refused(calls, lambda: c.store(0, k, k, ROWS), "is cut")
    c.plan(cu, ROWS)
    assert calls[-2][1][2] is c.kept
