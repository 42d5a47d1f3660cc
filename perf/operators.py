"""Paged keys and values, and the attention over prompts and pages, as timed cases.

Four operators of the library, each one pass through its public entry point:

  plan     seer_page_plan    pages taken and returned, block tables and slot map of a step
  store    seer_kv_store     key and value rows into their pages
  prompt   seer_attn_prompt  causal attention of packed prompts with grouped heads
  paged    seer_attn_paged   queries over pages: single tokens, trees of drafted tokens, causal chunks, windows

A pool is [pages, 2 (K | V), kv heads, slots of a page, head dim].  A case's fields:

  kind             one of the above
  dtype            bf16 | f32
  v16              whether V is held in fp16 beside bf16 keys, as the layer kernels leave it
  heads, kv, dim   query heads, key/value heads, head dim
  page             tokens of a page
  batch            requests
  past_lo, past_hi tokens of a request in the cache before the call
  new_lo, new_hi   rows of a request in the call
  drop             plan: up to this many of the cached tokens are given up (a cut window, refused drafts)
  ended            plan: every so manyeth request has ended and gives all its pages back, 0 for none
  mask             causal | tree | none
  pad              rows that the call's bound has past the last sequence
"""
import math

import torch

own = False

BASE = dict(dtype="bf16", v16=False, heads=32, kv=8, dim=128, page=64, batch=1, past_lo=0, past_hi=0, new_lo=1,
            new_hi=1, drop=0, ended=0, mask="causal", pad=0)


def _case(**changes):
    c = dict(BASE)
    c.update(changes)
    return c


def listed():
    return [
        # one decoding step of many requests: one token each, now and then one has ended
        _case(name="plan_decode", kind="plan", batch=256, past_lo=500, past_hi=8000, drop=3, ended=16),
        # windows cut at their boundaries give pages back while new windows of 1024 take theirs
        _case(name="plan_windows", kind="plan", page=16, batch=48, past_lo=800, past_hi=1817, new_lo=1024, new_hi=1024,
              drop=1000, ended=5, pad=256),
        # the keys and values of one token of each request
        _case(name="store_tokens", kind="store", batch=256, past_lo=500, past_hi=8000),
        # the prefixes of sixteen requests, from the rows that the layer leaves (V in fp16)
        _case(name="store_prefixes", kind="store", v16=True, kv=32, batch=16, new_lo=793, new_hi=1817, pad=100),
        # one short prompt in fp32: latency
        _case(name="prompt_f32_one", kind="prompt", dtype="f32", heads=4, kv=4, dim=64, new_lo=97, new_hi=97),
        # sixteen ragged prompts, as many key heads as query heads
        _case(name="prompt_b16", kind="prompt", heads=32, kv=32, batch=16, new_lo=200, new_hi=1300),
        # long prompts with grouped heads, the largest call
        _case(name="prompt_long", kind="prompt", batch=4, new_lo=1500, new_hi=8192),
        # short prompts of a small model: odd lengths, seven heads to a group, 64-wide heads
        _case(name="prompt_dim64", kind="prompt", heads=14, kv=2, dim=64, batch=9, new_lo=1, new_hi=700),
        # one request's next token: latency
        _case(name="paged_token_b1", kind="paged", past_lo=793, past_hi=793),
        # the next token of many requests with long contexts: the cache is read once
        _case(name="paged_tokens_b64", kind="paged", heads=28, kv=4, batch=64, past_lo=500, past_hi=16000),
        # trees of drafted tokens over the contexts of eight requests
        _case(name="paged_trees_b8", kind="paged", page=16, batch=8, past_lo=600, past_hi=4000, new_lo=24, new_hi=61,
              mask="tree"),
        # a denoising step's kept windows over the cached prefixes of sixteen requests, both ways (V in fp16)
        _case(name="paged_windows_b16", kind="paged", v16=True, heads=32, kv=32, batch=16, past_lo=793, past_hi=793,
              new_lo=35, new_hi=502, mask="none"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "store", "prompt", "prompt", "paged", "paged", "paged"])
    heads, kv, dim = rng.choice([(32, 8, 128), (32, 32, 128), (28, 4, 128), (14, 2, 64), (8, 8, 64), (16, 1, 128),
                                 (12, 4, 64)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if dtype == "f32":
        heads, kv, dim = rng.choice([(4, 4, 64), (8, 2, 128), (6, 3, 32), (8, 1, 80)])
    shape = dict(kind=kind, dtype=dtype, heads=heads, kv=kv, dim=dim, page=rng.choice([16, 32, 64, 128, 256]),
                 v16=dtype == "bf16" and rng.random() < 0.3, pad=rng.choice([0, 0, _log(rng, 1, 500)]))
    if kind == "plan":
        hi = _log(rng, 20, 16000)
        new = rng.choice([1, _log(rng, 1, 64), _log(rng, 64, 1024)])
        return _case(**dict(shape, batch=_log(rng, 1, 512 if new <= 64 else 40), past_lo=_log(rng, 1, hi), past_hi=hi,
                            new_lo=_log(rng, 1, new), new_hi=new, drop=rng.choice([0, 4, hi // 2]),
                            ended=rng.choice([0, 3, 10])))
    if kind == "store":
        if rng.random() < 0.5:
            hi = _log(rng, 20, 2000)
            return _case(**dict(shape, batch=_log(rng, 1, 256), past_lo=_log(rng, 1, hi), past_hi=hi))
        hi = _log(rng, 20, 1800)
        return _case(**dict(shape, batch=_log(rng, 1, 12), new_lo=_log(rng, 1, hi), new_hi=hi))
    if kind == "prompt":
        hi = _log(rng, 1, 1000 if dtype == "f32" else 5000)
        most = max(1, min(16, 12000 // hi))
        return _case(**dict(shape, batch=_log(rng, 1, most), new_lo=_log(rng, 1, hi), new_hi=hi))
    form = rng.choice(["token", "token", "tree", "chunk", "window"])
    past = _log(rng, 10, 16000 if dtype == "bf16" else 2000)
    shape.update(past_lo=_log(rng, 5, past), past_hi=past)
    if form == "token":
        return _case(**dict(shape, batch=_log(rng, 1, 64 if kv <= 8 else 24)))
    if form == "tree":
        new = _log(rng, 2, 150)
        return _case(**dict(shape, batch=_log(rng, 1, 16), new_lo=_log(rng, 1, new), new_hi=new, mask="tree"))
    past = min(past, 4000)
    new = _log(rng, 16, 800 if dtype == "bf16" else 200)
    return _case(**dict(shape, batch=_log(rng, 1, 10), past_lo=_log(rng, 5, past), past_hi=past, new_lo=_log(rng, 1, new),
                        new_hi=new, mask="causal" if form == "chunk" else "none"))


# ---- sizes ------------------------------------------------------------------------
def _spread(lo, hi, n, shift):
    """n whole numbers over [lo, hi], spread over their logarithm, in no order."""
    if lo >= hi:
        return [hi] * n
    at = [(0.5 + 0.6180339887498949 * i + shift) % 1.0 for i in range(n)]
    return [min(hi, max(lo, int(round(math.exp(math.log(max(lo, 0.5)) + a * math.log(hi / max(lo, 0.5))))))) for a in at]


def _sizes(case):
    """(tokens held before the call, tokens kept, rows of the call) of each request."""
    n = case["batch"]
    held = _spread(case["past_lo"], case["past_hi"], n, 0.0)
    new = _spread(case["new_lo"], case["new_hi"], n, 0.31)
    if n > 1:                                          # both ends of the range occur
        held[0], held[-1] = case["past_hi"], case["past_lo"]
        new[0], new[-1] = case["new_lo"], case["new_hi"]
    drop = [min(h, d) for h, d in zip(held, _spread(0, case["drop"], n, 0.77))]
    keep = [h - d for h, d in zip(held, drop)]
    if case["ended"]:
        for i in range(case["ended"] - 1, n, case["ended"]):
            keep[i], new[i] = 0, 0
    return held, keep, new


def _starts(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return out


def _types(case):
    if case["dtype"] == "f32":
        return torch.float32, torch.float32
    return torch.bfloat16, torch.float16 if case["v16"] else torch.bfloat16


def _ceil(a, b):
    return -(-a // b)


# ---- inputs -----------------------------------------------------------------------
def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    held, keep, new = _sizes(case)
    B, H, KV, D, ps, kind = case["batch"], case["heads"], case["kv"], case["dim"], case["page"], case["kind"]
    T = sum(new)
    rows = T + case["pad"]
    qt, vt = _types(case)

    def i32(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def normal(*shape):
        return torch.empty(shape, device="cuda", dtype=torch.float32).normal_(0.0, 1.0, generator=gen)

    a = dict(case=case, B=B, T=T, rows=rows, cu=i32(_starts(new)), new=i32(new))
    if kind in ("prompt", "store"):
        # rows of a projection, q | k | v side by side
        qkv = normal(rows, (H + 2 * KV) * D).to(qt)
        if vt != qt:
            qkv.view(vt)[:, (H + KV) * D:] = normal(rows, KV * D).to(vt)
        a["q"], a["k"], a["v"] = qkv[:, :H * D], qkv[:, H * D:(H + KV) * D], qkv.view(vt)[:, (H + KV) * D:]
    if kind == "prompt":
        a["out"] = torch.zeros(rows, H * D, dtype=qt, device="cuda")
        return a
    kv_len = [k + n for k, n in zip(keep, new)]
    full = [h if kind == "plan" else n for h, n in zip(held, kv_len)]      # tokens whose pages the table holds
    W = max(_ceil(max(h, n), ps) for h, n in zip(held, kv_len))
    most = sum(_ceil(max(h, n), ps) for h, n in zip(held, kv_len))
    P = most + most // 8 + 3
    ids = torch.randperm(P, generator=gen, device="cuda").to(torch.int32)
    pages = torch.tensor([_ceil(n, ps) for n in full], device="cuda")
    col = torch.arange(W, device="cuda")[None, :]
    base = torch.cumsum(pages, 0) - pages
    a["table"] = torch.where(col < pages[:, None], ids[(base[:, None] + col).clamp(max=P - 1)], -1).to(torch.int32)
    a.update(W=W, P=P, kv_len=i32(kv_len))
    if kind == "plan":
        used = sum(_ceil(n, ps) for n in full)
        a["free"] = torch.cat([ids[used:], torch.full((used,), -1, dtype=torch.int32, device="cuda")])
        a.update(held=i32(held), keep=i32(keep), free_in=i32([P - used]), free_out=i32([0]), status=i32([0]),
                 slots=torch.zeros(rows, dtype=torch.int32, device="cuda"))
        return a
    pool = normal(P, 2, KV, ps, D).to(qt)
    if vt != qt:
        pool.view(vt)[:, 1] = pool[:, 1].to(vt)
    a["pool"] = pool
    if kind == "store":
        r = torch.arange(T, device="cuda")
        b = torch.searchsorted(a["cu"][1:].contiguous(), r.to(torch.int32), right=True)
        pos = i32(keep)[b] + r - a["cu"][b]
        a["slots"] = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        a["slots"][:T] = a["table"][b, pos // ps] * ps + (pos % ps).to(torch.int32)
        return a
    a["q"] = normal(rows, H * D).to(qt)
    a["out"] = torch.zeros(rows, H * D, dtype=qt, device="cuda")
    if case["mask"] == "tree":
        # each drafted token hangs on one of the few before it, or on the context; it sees its ancestors and itself
        n = max(new)
        words = _ceil(n, 64)
        pick = torch.randint(1, 9, (B, n), generator=gen, device="cuda").cpu().tolist()
        bits = []
        for i in range(B):
            seen = []
            for j in range(new[i]):
                up = j - pick[i][j]
                seen.append((seen[up] if up >= 0 else 0) | 1 << j)
            bits += [[(m >> 64 * w & 0xffffffffffffffff) - (m >> 64 * w + 63 & 1) * (1 << 64) for w in range(words)]
                     for m in seen]
        a["bits"] = torch.zeros(rows, words, dtype=torch.int64, device="cuda")
        a["bits"][:T] = torch.tensor(bits, dtype=torch.int64, device="cuda")
    return a


def _bytes(n):
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    a = _inputs(case, seed)
    if own:
        from paper_2607_14557_amd import seer as S
        a["desc"] = S.seer_attn_desc(case["heads"], case["kv"], case["dim"],
                                     S.SEER_DTYPE_BF16 if case["dtype"] == "bf16" else S.SEER_DTYPE_F32,
                                     S.SEER_ATTN_V_F16 if case["v16"] else 0, 0.0)
        if case["kind"] != "prompt":
            a["pages"] = S.seer_page_desc(case["page"], a["P"], a["W"])
        if case["kind"] in ("prompt", "paged"):
            a["ws"] = _bytes(S.seer_attn_workspace_bytes(a["desc"], a["rows"], a["B"]))
    return a


# ---- the plain forms, in 32 bits ----------------------------------------------------
def _plain_plan(a):
    case, B, W, P, ps = a["case"], a["B"], a["W"], a["P"], a["case"]["page"]
    held, keep, new, cu = a["held"].long(), a["keep"].long(), a["new"].long(), a["cu"].long()
    table, free, count = a["table"].clone(), a["free"].clone(), a["free_in"].long()
    H, N = (held + ps - 1) // ps, (keep + new + ps - 1) // ps
    give, take = (H - N).clamp(min=0), (N - H).clamp(min=0)
    gave, took = give.sum(), take.sum()
    col = torch.arange(W, device=table.device)[None, :]
    # returned pages in request order, then in column order; cells that return none go to the place behind them all
    at = torch.cumsum(give, 0)[:, None] - give[:, None] + col - N[:, None]
    back = torch.full((P + 1,), -1, dtype=torch.int32, device=table.device)
    back[torch.where((col >= N[:, None]) & (col < H[:, None]), at, P).flatten()] = table.flatten()
    # the stack of free pages with the returned ones on top; the k-th page taken comes from k below its top
    k = torch.cumsum(take, 0)[:, None] - take[:, None] + col - H[:, None]
    pos = count + gave - 1 - k
    got = torch.where(pos < count, free[pos.clamp(0, P - 1)], back[(pos - count).clamp(0, P)])
    table = torch.where((col >= H[:, None]) & (col < N[:, None]), got, table)
    place = torch.arange(P, device=table.device)
    free = torch.where((place >= count) & (place < count + gave - took), back[(place - count).clamp(0, P)], free)
    r = torch.arange(a["rows"], device=table.device)
    b = torch.searchsorted(cu[1:].contiguous(), r, right=True).clamp(max=B - 1)
    pos = (keep[b] + r - cu[b]).clamp(min=0)
    slots = table[b, (pos // ps).clamp(max=W - 1)].long() * ps + pos % ps
    slots = torch.where(r < cu[B], slots, -1)
    return {"table": table, "kv_len": (keep + new).int(), "slots": slots.int(), "free": free,
            "free_out": (count + gave - took).int(), "status": torch.zeros_like(a["status"])}


def _plain_store(a):
    case, T, ps = a["case"], a["T"], a["case"]["page"]
    slot = a["slots"][:T].long()
    for half, rows in enumerate((a["k"], a["v"])):
        a["pool"].view(rows.dtype)[slot // ps, half, :, slot % ps] = rows[:T].view(T, case["kv"], case["dim"])
    return _pool(a)


def _pool(a):
    vt = _types(a["case"])[1]
    return {"k": a["pool"][:, 0], "v": a["pool"].view(vt)[:, 1]}


def _padded(x, cu, n, width):
    """[batch, width, ...] from packed rows; places past a sequence hold some row of the batch."""
    at = cu[:-1, None].long() + torch.arange(width, device=x.device)[None, :]
    return x[at.clamp(max=max(0, n - 1))]


def _attend(case, q, k, v, seen):
    """q [B, n, heads, dim], k and v [B, L, kv, dim], seen [B, 1, n, L]: softmax attention in 32 bits, zero where a
    query sees nothing."""
    B, n, H, D = q.shape
    KV, G = case["kv"], case["heads"] // case["kv"]
    q = q.float().view(B, n, KV, G, D).permute(0, 2, 1, 3, 4).reshape(B, KV, n * G, D)
    k = k.float().permute(0, 2, 3, 1).contiguous()
    v = torch.where(torch.isfinite(v), v, 0).float().permute(0, 2, 1, 3).contiguous()
    s = torch.matmul(q, k).view(B, KV, n, G, -1) * D ** -0.5
    s = s.masked_fill_(~seen[:, :, :, None, :], -math.inf)
    p = torch.exp(s.sub_(s.amax(-1, keepdim=True).clamp(min=-3e38)))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, KV, n * G, -1), v).view(B, KV, n, G, D)
    o = torch.where(total > 0, o / total, 0)
    return o.permute(0, 2, 1, 3, 4).reshape(B, n, H, D)


def _unpadded(a, o):
    """The rows of the call, packed, from [batch, width, heads, dim], in the output's buffer."""
    case, T = a["case"], a["T"]
    r = torch.arange(T, device=o.device)
    b = torch.searchsorted(a["cu"][1:].contiguous(), r.int(), right=True)
    a["out"][:T] = o[b, r - a["cu"].long()[b]].reshape(T, -1).to(a["out"].dtype)
    return a["out"]


def _plain_prompt(a):
    case, T = a["case"], a["T"]
    H, KV, D = case["heads"], case["kv"], case["dim"]
    n = case["new_hi"]
    q, k, v = (_padded(x[:T], a["cu"], T, n).view(a["B"], n, h, D) for x, h in ((a["q"], H), (a["k"], KV), (a["v"], KV)))
    at = torch.arange(n, device=q.device)
    seen = (at[None, :] <= at[:, None])[None, None] & (at < a["new"][:, None])[:, None, None, :]
    return _unpadded(a, _attend(case, q, k, v, seen))


def _plain_paged(a):
    case, T, B, ps = a["case"], a["T"], a["B"], a["case"]["page"]
    H, D, n = case["heads"], case["dim"], case["new_hi"]
    L = case["past_hi"] + n
    at = torch.arange(L, device="cuda")
    page = a["table"][:, (at // ps).clamp(max=a["W"] - 1)].long().clamp(min=0)
    k = a["pool"][page, 0, :, (at % ps)[None, :]]
    v = a["pool"].view(_types(case)[1])[page, 1, :, (at % ps)[None, :]]
    q = _padded(a["q"][:T], a["cu"], T, n).view(B, n, H, D)
    past = (a["kv_len"] - a["new"])[:, None, None, None]
    row = torch.arange(n, device="cuda")[None, None, :, None]
    seen = (at < a["kv_len"][:, None])[:, None, None, :].expand(B, 1, n, L)
    if case["mask"] == "causal":
        seen = seen & (at <= past + row)
    if case["mask"] == "tree":
        bits = _padded(a["bits"][:T], a["cu"], T, n)[:, None]                      # [B, 1, n, words]
        j = (at - past).clamp(min=0, max=64 * bits.shape[-1] - 1).expand(B, 1, n, L)
        seen = seen & ((at < past) | (torch.gather(bits, 3, j // 64) >> (j % 64) & 1).bool())
    return _unpadded(a, _attend(case, q, k, v, seen))


# ---- one pass -----------------------------------------------------------------------
def run(a):
    case, kind = a["case"], a["case"]["kind"]
    if not own:
        return {"plan": _plain_plan, "store": _plain_store, "prompt": _plain_prompt, "paged": _plain_paged}[kind](a)
    from paper_2607_14557_amd import seer as S
    if kind == "plan":
        S.seer_page_plan(a["pages"], a["held"], a["keep"], a["cu"], None, a["B"], a["rows"], a["free"], a["free_in"],
                         a["free_out"], a["table"], a["kv_len"], a["slots"], a["status"])
        return {n: a[n] for n in ("table", "kv_len", "slots", "free", "free_out", "status")}
    if kind == "store":
        S.seer_kv_store(a["desc"], a["pages"], a["k"], a["k"].stride(0), a["v"], a["v"].stride(0), a["rows"],
                        a["slots"], a["pool"])
        return _pool(a)
    if kind == "prompt":
        S.seer_attn_prompt(a["desc"], S.SEER_MASK_CAUSAL, a["q"], a["q"].stride(0), a["k"], a["k"].stride(0), a["v"],
                           a["v"].stride(0), a["out"], a["out"].stride(0), a["rows"], a["cu"], None, a["B"], a["ws"])
        return a["out"]
    mask = {"none": S.SEER_MASK_NONE, "causal": S.SEER_MASK_CAUSAL, "tree": S.SEER_MASK_TREE}[case["mask"]]
    bits = a.get("bits")
    S.seer_attn_paged(a["desc"], a["pages"], mask, a["q"], a["q"].stride(0), a["out"], a["out"].stride(0), a["rows"],
                      a["cu"], None, a["B"], a["pool"], a["table"], a["kv_len"], bits,
                      0 if bits is None else bits.shape[1], a["ws"])
    return a["out"]


# ---- what a pass cannot do without ----------------------------------------------------
def work(case):
    held, keep, new = _sizes(case)
    B, H, KV, D, ps, T = case["batch"], case["heads"], case["kv"], case["dim"], case["page"], sum(new)
    es = 2 if case["dtype"] == "bf16" else 4
    kv_len = [k + n for k, n in zip(keep, new)]
    if case["kind"] == "plan":
        moved = sum(abs(_ceil(h, ps) - _ceil(n, ps)) for h, n in zip(held, kv_len))
        # lengths in and out, one entry read and one written for each page that moves, a slot for each row
        return {"bytes": 4.0 * (4 * B + 2 * moved + sum(_ceil(n, ps) for n in new) + T + case["pad"]), "flops": 0.0}
    if case["kind"] == "store":
        return {"bytes": 2.0 * T * 2 * KV * D * es + 4.0 * T, "flops": 0.0}
    if case["kind"] == "prompt":
        pairs = sum(n * (n + 1) / 2 for n in new)
        return {"bytes": T * (2.0 * H + 2.0 * KV) * D * es, "flops": 4.0 * D * H * pairs}
    if case["mask"] == "causal":
        pairs = sum(n * k + n * (n + 1) / 2 for n, k in zip(new, keep))
    else:
        pairs = sum(n * (k + n) for n, k in zip(new, keep))
    return {"bytes": 2.0 * T * H * D * es + 2.0 * sum(kv_len) * KV * D * es + 4.0 * sum(_ceil(n, ps) for n in kv_len),
            "flops": 4.0 * D * H * pairs}


# ---- the definition in 64 bits ----------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "plan":
        return None                                   # whole numbers
    a = _inputs(case, seed)
    held, keep, new = _sizes(case)
    H, KV, D, ps = case["heads"], case["kv"], case["dim"], case["page"]
    if case["kind"] == "store":
        k, v = a["pool"][:, 0].double(), a["pool"].view(a["v"].dtype)[:, 1].double()
        r = 0
        for b, n in enumerate(new):
            for first in range(keep[b] - keep[b] % ps, keep[b] + n, ps):       # the pages that rows go to
                lo, hi = max(first, keep[b]), min(first + ps, keep[b] + n)
                page, rows = a["table"][b, first // ps], slice(r + lo - keep[b], r + hi - keep[b])
                for to, rows in ((k, a["k"][rows]), (v, a["v"][rows])):
                    to[page, :, lo - first:hi - first] = rows.double().view(hi - lo, KV, D).transpose(0, 1)
            r += n
        return {"k": k, "v": v}
    out = torch.zeros(a["rows"], H * D, dtype=torch.float64, device="cuda")
    bits = a["bits"].cpu().tolist() if case["kind"] == "paged" and case["mask"] == "tree" else None
    r0 = 0
    for b, n in enumerate(new):
        past = keep[b] if case["kind"] == "paged" else 0
        L = past + n
        seen = torch.ones(n, L, dtype=torch.bool, device="cuda")
        if case["mask"] == "causal":
            seen = torch.tril(seen, diagonal=past)
        elif bits is not None:
            rows = [[bits[r0 + i][j // 64] >> (j % 64) & 1 for j in range(n)] for i in range(n)]
            seen[:, past:] = torch.tensor(rows, dtype=torch.bool, device="cuda")
        if case["kind"] == "prompt":
            k, v = a["k"][r0:r0 + n].view(n, KV, D), a["v"][r0:r0 + n].view(n, KV, D)
        else:
            pages = a["table"][b, :_ceil(L, ps)].long()
            k = a["pool"][pages, 0].transpose(1, 2).reshape(-1, KV, D)[:L]
            v = a["pool"].view(_types(case)[1])[pages, 1].transpose(1, 2).reshape(-1, KV, D)[:L]
        for h in range(H):
            kh, vh = k[:, h * KV // H].double(), v[:, h * KV // H].double()
            for i in range(0, n, 2048):
                qh = a["q"][r0 + i:r0 + min(n, i + 2048), h * D:(h + 1) * D].double()
                s = (qh @ kh.t().contiguous() / math.sqrt(D)).masked_fill(~seen[i:i + 2048], -math.inf)
                out[r0 + i:r0 + min(n, i + 2048), h * D:(h + 1) * D] = torch.softmax(s, dim=1) @ vh
        r0 += n
    return out
