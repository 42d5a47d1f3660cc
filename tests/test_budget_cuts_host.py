"""What BudgetCache hands to its calls around a cut (no GPU): the lengths that a plan keeps, recorded or not, and what it
refuses before anything is launched or changed."""
import ctypes
import os

import pytest
import torch

from test_budget_host import B, CALLS, D, FAKE, H, KV, ROWS, _bf16, _i32, rope


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    if not os.path.exists(seer.LIB_PATH):
        pytest.skip("libseer.so not built")
    seer.load_library()
    return seer


@pytest.fixture
def calls(S, monkeypatch):
    """The entry points' names, arguments and keywords as they are called, with no launch behind them."""
    from paper_2607_14557_amd import runner
    made = []
    for name in CALLS:
        monkeypatch.setattr(runner.S, name, lambda *a, _name=name, **kw: made.append((_name, a, kw)))
    return made


def _cache(S, layers=2, **kw):
    from paper_2607_14557_amd.runner import BudgetCache
    return BudgetCache(H, KV, D, layers, 4, 16, B, 32, ROWS, rope=rope(S), device="cpu", **kw)


def _plans(calls):
    return [(a, kw) for n, a, kw in calls if n == "seer_page_plan_latched"]


def _positions(calls):
    return [(a, kw) for n, a, kw in calls if n == "seer_row_positions"]


def test_what_a_plan_keeps(S, calls):
    """One array, whatever came before on the host: a call that is recorded is made once and replayed in other states."""
    c, cu, budget = _cache(S), _i32(B + 1), _i32(B)
    c.plan(cu, ROWS)                                    # nothing is cut
    for _ in range(2):                                  # as two steps are recorded
        c.plan(cu, ROWS)
        for layer in range(2):
            c.evict(layer, budget)
    c.plan(cu, ROWS)                                    # behind the recording, of which nothing has run
    plans, after = _plans(calls), _positions(calls)
    assert len(plans) == 4 and all(a[2] is c.kept for a, _ in plans)
    # and it is the lengths of an accepted plan from then on: each after its plan, with its status
    order = [n for n, _, _ in calls if n in ("seer_page_plan_latched", "seer_row_positions")]
    assert order == ["seer_page_plan_latched", "seer_row_positions"] * 4
    for (a, _), (pa, pkw) in zip(plans, after):
        assert pkw["kept"] is c.kept and pkw["kv_len"] is a[11] and pa[5] is a[13]


def test_plan_keeps_apart_what_it_writes(S, calls):
    c, cu, budget = _cache(S), _i32(B + 1), _i32(B)
    whole = c.kept = _i32(3 * B)[:B]                    # kept within something larger
    parts = whole.as_strided((B,), (1,), whole.storage_offset())
    for kw in (dict(base=c.kept), dict(base=parts), dict(seqused=c.kept),
               dict(base=whole.as_strided((B,), (1,), whole.storage_offset() + B - 1))):
        before, lens, seen = len(calls), c._lens[0], c._seen[0]
        with pytest.raises(ValueError, match="writes"):
            c.plan(cu, ROWS, **kw)
        assert len(calls) == before and c._lens[0] is lens and c._seen[0] is seen
    c.plan(cu, ROWS, base=whole.as_strided((B,), (1,), whole.storage_offset() + B))
    c.plan(cu, ROWS, c.kept)                            # read by the plan, written behind it


def test_row_positions_kept_refusals(S):
    def call(cu=FAKE, used=None, batch=2, seen=FAKE, base=None, status=None, rows=4, pos=FAKE, next=2 * FAKE, kv=3 * FAKE,
             kept=4 * FAKE):
        return S.load_library().seer_row_positions_kept(cu, used, batch, seen, base, status, rows, pos, next, kv, kept, None)

    for kw in (dict(cu=None), dict(pos=None), dict(batch=0), dict(rows=-1), dict(next=FAKE), dict(kv=None), dict(kept=None)):
        assert call(**kw) == S.SEER_EINVAL, kw
    for kw in (dict(kept=FAKE), dict(kept=2 * FAKE), dict(kept=3 * FAKE), dict(used=4 * FAKE), dict(base=4 * FAKE),
               dict(status=4 * FAKE)):
        assert call(**kw) == S.SEER_EINVAL and "kept" in S.seer_last_error(), kw
    assert ctypes.c_int(call(rows=0, pos=None, batch=0)).value == S.SEER_EINVAL


def test_layers_of_one_cut(S, calls):
    """The layers after the first are held to what the first one keeps."""
    c, cu, budget = _cache(S, layers=3), _i32(B + 1), _i32(B)
    for shared in (False, True):
        c.plan(cu, ROWS)
        for layer in (1, 0, 2):
            c.evict(layer, budget, shared=shared)
        one = S.SEER_EVICT_SHARED if shared else 0
        cuts = [a for n, a, _ in calls if n == "seer_kv_evict"][-3:]
        assert [a[2] for a in cuts] == [one, one | S.SEER_EVICT_ALIKE, one | S.SEER_EVICT_ALIKE]
        assert all(a[15] is c.kept for a in cuts)


def test_what_bounds_a_keep(S, calls):
    """A plan knows what the cut has left, whoever says what stays."""
    c, cu, keep = _cache(S, layers=1), _i32(B + 1), _i32(B)
    for k in (None, keep):
        c.plan(cu, ROWS, k)
        c.evict(0, keep)
    assert all(kw["kept"] is c.kept for _, kw in _plans(calls)) and _plans(calls)[1][0][2] is keep


def test_page_plan_kept_refusals(S):
    names = ("held", "kept", "keep", "cu", "used", "batch", "rows", "free", "free_in", "free_out", "table", "kv", "slots",
             "status", "refused")

    def call(**kw):
        a = dict(held=FAKE, kept=2 * FAKE, keep=2 * FAKE, cu=FAKE, used=None, batch=2, rows=4, free=FAKE, free_in=FAKE,
                 free_out=3 * FAKE, table=FAKE, kv=4 * FAKE, slots=FAKE, status=FAKE, refused=5 * FAKE)
        a.update(kw)
        return S.load_library().seer_page_plan_kept(ctypes.byref(S.seer_page_desc(64, 100, 10)), *[a[n] for n in names], None)

    for n in ("held", "kept", "keep", "cu", "free", "free_in", "free_out", "table", "kv", "slots", "status", "refused"):
        assert call(**{n: None}) == S.SEER_EINVAL, n
    for kw in (dict(kv=2 * FAKE, keep=FAKE), dict(kv=FAKE), dict(free_out=FAKE), dict(refused=FAKE), dict(batch=0), dict(rows=-1)):
        assert call(**kw) == S.SEER_EINVAL, kw
    assert call(batch=4097) == S.SEER_EUNSUPPORTED


def test_base_within_what_a_plan_writes(S, calls):
    """A view of the buffer is the buffer: refused before the pages are planned and the lengths change places."""
    c, cu = _cache(S), _i32(B + 1)
    for n in range(2):
        old = c._seen[1]
        assert old is not c.seen
        for kw in (dict(base=old), dict(base=old[:]), dict(base=old.view(B)), dict(seqused=old)):
            before, lens, seen = len(calls), c._lens[0], c._seen[0]
            with pytest.raises(ValueError, match="writes"):
                c.plan(cu, ROWS, **kw)
            assert len(calls) == before and c._lens[0] is lens and c._seen[0] is seen and c._planned == n * ROWS
        c.plan(cu, ROWS, base=c.seen[:])


def test_evict_knows_the_plan(S, calls):
    c, cu, budget = _cache(S), _i32(B + 1), _i32(B)
    c.plan(cu, ROWS)
    c.evict(0, budget)
    assert calls[-1][0] == "seer_kv_evict" and calls[-1][2]["status"] is c.status and calls[0][1][13] is c.status


def test_evict_planned_refusals(S):
    names = ("flags", "kv", "budget", "seen", "batch", "first", "recent", "table", "pool", "weight", "number", "wo", "no",
             "kept", "status", "ws", "bytes")

    def call(**kw):
        a = dict(flags=0, kv=FAKE, budget=2 * FAKE, seen=3 * FAKE, batch=2, first=0, recent=0, table=FAKE, pool=FAKE,
                 weight=FAKE, number=2 * FAKE, wo=FAKE, no=2 * FAKE, kept=4 * FAKE, status=5 * FAKE, ws=FAKE, bytes=1 << 40)
        a.update(kw)
        return S.load_library().seer_kv_evict_planned(ctypes.byref(S.seer_attn_desc(8, 2, 128, S.SEER_DTYPE_BF16, 0, 0.0)),
                                                      ctypes.byref(S.seer_page_desc(64, 100, 10)), *[a[n] for n in names], None)

    for n in ("kv", "budget", "seen", "table", "pool", "weight", "number", "wo", "no", "kept", "status", "ws"):
        assert call(**{n: None}) == S.SEER_EINVAL, n
    for kw in (dict(status=4 * FAKE), dict(flags=2), dict(flags=8), dict(batch=0), dict(kept=FAKE), dict(bytes=16, flags=4)):
        assert call(**kw) in (S.SEER_EINVAL, S.SEER_EWORKSPACE), kw


def test_rope_that_is_none(S, calls):
    """Rows that do not turn have neither a description nor frequencies; one without the other is refused."""
    from paper_2607_14557_amd.runner import BudgetCache
    c, cu = BudgetCache(H, KV, D, 1, 4, 16, B, 32, ROWS, device="cpu"), _i32(B + 1)
    c.plan(cu, ROWS)
    c.store(0, _bf16(ROWS, KV * D), _bf16(ROWS, KV * D), ROWS)
    c.rotate(_bf16(ROWS, H * D), None, ROWS)
    assert calls[-2][0] == "seer_kv_store_rope" and calls[-2][1][2:4] == (None, None)
    assert calls[-1][0] == "seer_rope_rows" and calls[-1][1][1:3] == (None, None)
    L, d, p = S.load_library(), S.seer_attn_desc(H, KV, D, S.SEER_DTYPE_BF16, 0, 0.0), S.seer_page_desc(16, 4, 2)
    r = rope(S)
    for desc, turns in ((None, FAKE), (ctypes.byref(r), None)):
        assert L.seer_rope_rows(ctypes.byref(d), desc, turns, 0, FAKE, 256, None, 0, FAKE, 256, None, 0, 4, FAKE, None) == S.SEER_EINVAL
        assert "go together" in S.seer_last_error()
        assert L.seer_kv_store_rope(ctypes.byref(d), ctypes.byref(p), desc, turns, None, 0, None, 0, FAKE, 128, FAKE, 128, 4, FAKE,
                                    FAKE, FAKE, FAKE, FAKE, None) == S.SEER_EINVAL
    # without either, the other checks stand
    assert L.seer_rope_rows(ctypes.byref(d), None, None, 0, FAKE, 256, None, 0, FAKE, 256, None, 0, 4, None, None) == S.SEER_EINVAL
    assert L.seer_kv_store_rope(ctypes.byref(d), ctypes.byref(p), None, None, None, 0, None, 0, FAKE, 128, FAKE, 128, 4, FAKE,
                                None, FAKE, FAKE, FAKE, None) == S.SEER_EINVAL


def test_budget_within_kept(S, calls):
    """The lengths that the layers before keep may be the budget of the next one; part of them, moved, may not."""
    c, cu = _cache(S), _i32(B + 1)
    whole = c.kept = _i32(3 * B)[:B]
    c.plan(cu, ROWS)
    c.evict(0, _i32(B))
    c.evict(1, c.kept)
    assert calls[-1][1][4] is c.kept and calls[-1][1][2] == S.SEER_EVICT_ALIKE
    c.plan(cu, ROWS)
    with pytest.raises(ValueError, match="budget"):
        c.evict(0, whole.as_strided((B,), (1,), whole.storage_offset() + 1))
    c.evict(0, whole.as_strided((B,), (1,), whole.storage_offset() + B))
