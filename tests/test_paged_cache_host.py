"""What PagedCache takes and refuses (no GPU): types, rows, strides and sizes that the kernels would read past an end
or take for something else."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def S():
    from paper_2607_14557_amd import seer
    if not os.path.exists(seer.LIB_PATH):
        pytest.skip("libseer.so not built")
    seer.load_library()
    return seer


@pytest.fixture
def calls(S, monkeypatch):
    """The entry points' names as they are called, with no launch behind them."""
    from paper_2607_14557_amd import runner
    made = []
    for name in ("seer_page_plan_latched", "seer_kv_store", "seer_attn_paged", "seer_attn_prompt"):
        monkeypatch.setattr(runner.S, name, lambda *a, _name=name, **kw: made.append((_name, a)))
    return made


H, KV, D, B, ROWS = 4, 2, 64, 3, 8


def _cache(**kw):
    from paper_2607_14557_amd.runner import PagedCache
    return PagedCache(H, KV, D, 1, 4, 16, B, 32, ROWS, device="cpu", **kw)


def _i32(n):
    return torch.zeros(n, dtype=torch.int32)


def _bf16(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def _refused(calls, call, match):
    before = len(calls)
    with pytest.raises(ValueError, match=match):
        call()
    assert len(calls) == before


def test_arrays_of_requests(calls):
    c, cu = _cache(), _i32(B + 1)
    q, k = _bf16(ROWS, H * D), _bf16(ROWS, KV * D)
    for bad in (cu.long(), cu.float(), _i32(2 * B + 2)[::2]):
        _refused(calls, lambda: c.plan(bad, ROWS), "cu")
        _refused(calls, lambda: c.attend(0, q, q.clone(), bad, ROWS), "cu")
        _refused(calls, lambda: c.prompt(q, k, k, q.clone(), bad, ROWS), "cu")
    for bad in (_i32(B).long(), _i32(2 * B)[::2]):
        _refused(calls, lambda: c.plan(cu, ROWS, bad), "keep")
        _refused(calls, lambda: c.plan(cu, ROWS, None, bad), "seqused")
        _refused(calls, lambda: c.attend(0, q, q.clone(), cu, ROWS, seqused=bad), "seqused")
    c.plan(cu, ROWS, _i32(B), _i32(B + 5))
    assert [n for n, _ in calls] == ["seer_page_plan_latched"]


def test_slots(calls):
    c, k = _cache(), _bf16(ROWS, KV * D)
    c.plan(_i32(B + 1), ROWS)
    for bad in (_i32(ROWS - 1), _i32(ROWS).long(), _i32(2 * ROWS)[::2]):
        _refused(calls, lambda: c.store(0, k, k, ROWS, bad), "slots")
    c.store(0, k, k, ROWS, _i32(ROWS))
    c.store(0, k, k, ROWS)
    assert len(calls) == 3


@pytest.mark.parametrize("v_f16", [False, True])
def test_rows(calls, v_f16):
    c, cu = _cache(v_f16=v_f16), _i32(B + 1)
    q, k = _bf16(ROWS, H * D), _bf16(ROWS, KV * D)
    v = k.half() if v_f16 else k
    for bad in (q[:ROWS - 1], q[:, :H * D - 8], q.float(), q.half(), _bf16(H * D, ROWS).t(), _bf16(ROWS, 2 * H * D)[:, ::2],
                q.view(ROWS, D, H).transpose(1, 2), q[0],
                q.view(ROWS, H // 2, 2, D).transpose(1, 2), _bf16(ROWS, H, 2 * D)[:, :, :D]):
        _refused(calls, lambda: c.attend(0, bad, q, cu, ROWS), "q ")
        _refused(calls, lambda: c.attend(0, q, bad, cu, ROWS), "out ")
        _refused(calls, lambda: c.prompt(bad, k, v, q, cu, ROWS), "q ")
        _refused(calls, lambda: c.prompt(q, k, v, bad, cu, ROWS), "out ")
    c.plan(cu, ROWS)
    for bad in (k[:ROWS - 1], k[:, 8:], k.float(), _bf16(ROWS, 2 * KV * D)[:, ::2]):
        _refused(calls, lambda: c.store(0, bad, v, ROWS), "k ")
        _refused(calls, lambda: c.prompt(q, bad, v, q.clone(), cu, ROWS), "k ")
    for bad in (v[:ROWS - 1], v[:, 8:], v.float(), k if v_f16 else k.half()):
        _refused(calls, lambda: c.store(0, k, bad, ROWS), "v ")
        _refused(calls, lambda: c.prompt(q, k, bad, q.clone(), cu, ROWS), "v ")
    del calls[:]
    # what the documentation allows: columns of a wider buffer, heads as a dimension, more rows, fewer of them in use
    qkv = _bf16(ROWS + 5, (H + 2 * KV) * D)
    c.attend(0, qkv[:, :H * D], q.view(ROWS, H, D), cu, ROWS)
    c.attend(0, qkv, q, cu, 1)
    c.store(0, qkv[:, H * D:(H + KV) * D], v.view(ROWS, KV, D), ROWS)
    c.prompt(qkv[:, :H * D], qkv[:, H * D:(H + KV) * D], v, q, cu, ROWS)
    c.attend(0, q.view(ROWS, KV, H // KV, D), qkv.view(ROWS + 5, H + 2 * KV, D)[:, :H], cu, ROWS)
    assert len(calls) == 5


def test_tree_bits(calls, S):
    c, cu, q = _cache(), _i32(B + 1), _bf16(ROWS, H * D)
    wide = torch.zeros(ROWS, 3, dtype=torch.int64)
    for bad in (wide[:, :1], wide[:ROWS - 1], wide.int(), wide[:, 0], wide[::2], wide.t()):
        _refused(calls, lambda: c.attend(0, q, q.clone(), cu, ROWS, S.SEER_MASK_TREE, bad), "tree_bits")
    c.attend(0, q, q.clone(), cu, ROWS, S.SEER_MASK_TREE, wide)
    assert len(calls) == 1 and calls[0][1][15] == 3


def test_a_store_of_more_rows_than_were_planned(calls):
    """Slots behind the last plan's rows are an earlier plan's: they would overwrite its tokens."""
    c, k, cu = _cache(), _bf16(ROWS, KV * D), _i32(B + 1)
    _refused(calls, lambda: c.store(0, k, k, 1), "last plan")
    c.plan(cu, ROWS)
    c.store(0, k, k, ROWS)
    slots = c.plan(cu, 2)
    for call in (lambda: c.store(0, k, k, 3), lambda: c.store(0, k, k, ROWS, slots), lambda: c.store(0, k, k, 3, c.slots)):
        _refused(calls, call, "last plan")
    c.store(0, k, k, 2)
    c.store(0, k, k, 1, slots)
    c.store(0, k, k, ROWS, _i32(ROWS))                # slots of the caller's own
    assert [n for n, _ in calls] == ["seer_page_plan_latched", "seer_kv_store"] * 2 + ["seer_kv_store"] * 2


def test_check_takes_a_raw_handle(calls, S, monkeypatch):
    """As every other call does: 0 is the default stream, whatever the current one is."""
    waited = []

    class Stream:
        def __init__(self, name):
            self.name = name

        def synchronize(self):
            waited.append(self.name)

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream("current"))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream("default"))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream(handle))
    c = _cache()
    for s in (None, 0, 12345, Stream("own")):
        c.check(s)
    assert waited == ["current", "default", 12345, "own"]
    c.refused.fill_(S.SEER_PAGES_WIDTH)
    with pytest.raises(S.SeerError):
        c.check(12345)
    c.check(12345)                                    # raised once


def test_latched_plan_refusals(S):
    fake = 1 << 20
    args = [fake, fake + 4096, fake, None, 2, 10, fake, fake, fake + 256, fake, fake + 8192, fake, fake]
    pages = ctypes.byref(S.seer_page_desc(64, 100, 10))
    call = S.load_library().seer_page_plan_latched
    assert call(pages, *args, None, None) == S.SEER_EINVAL
    assert call(pages, *args, fake, None) == S.SEER_EINVAL and "refused" in S.seer_last_error()
    assert call(pages, *(args[:4] + [0] + args[5:]), fake + 512, None) == S.SEER_EINVAL and "batch" in S.seer_last_error()
