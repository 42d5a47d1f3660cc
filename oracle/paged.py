"""Keys and values of many requests in pages, and the attention over them
(oracle, plain Python and fp64).

The paper combines its truncation with a KV cache (Appendix D, compatibility
with KV caching) and says nothing of how the cache is held.  Reading: pages of
a fixed number of tokens from one pool, a row of page numbers per request, and
a stack of free pages.  A step keeps the first tokens of each request, gives
the pages behind them back (a window cut at its boundary, refused drafts, an
ended request) and takes pages for its new rows.

Attention (Sec. 3.6 equations, with grouped heads: query head h reads
key/value head h // (heads // kv heads)) over the keys that a row sees: all of
its request's, those up to its own position, or the context and the rows of
the call that its bits name.  Keys that a row does not see are not computed
with at all.
"""
import numpy as np

EXHAUSTED, WIDTH, INVALID = 1, 2, 4


def pages_of(tokens, page):
    return -(-int(tokens) // page)


def plan(held, keep, lens, used, table, free, page, n_pages, rows_ub):
    """One step of the page book-keeping.  held, keep, lens (rows of the call),
    used (real rows; None: all) per request; table: list of lists; free: the
    stack, top last.  Returns dict(table, free, kv_len, slots, status); the
    arguments are not changed."""
    used = list(lens) if used is None else [max(0, min(u, n)) for u, n in zip(used, lens)]
    width = len(table[0])
    status = 0
    for h, k, n in zip(held, keep, used):
        if h < 0 or k < 0 or k > h or pages_of(max(h, 0), page) > width:
            status |= INVALID
        if pages_of(k + n, page) > width:
            status |= WIDTH
    refused = dict(table=[list(t) for t in table], free=list(free), kv_len=list(held), slots=[-1] * rows_ub)
    if status:
        return dict(refused, status=status)
    new, stack = [list(t) for t in table], list(free)
    for b, (h, k, n) in enumerate(zip(held, keep, used)):
        for e in range(pages_of(k + n, page), pages_of(h, page)):
            stack.append(table[b][e])
    if len(stack) > n_pages:
        return dict(refused, status=INVALID)
    for b, (h, k, n) in enumerate(zip(held, keep, used)):
        for e in range(pages_of(h, page), pages_of(k + n, page)):
            if not stack:
                return dict(refused, status=EXHAUSTED)
            new[b][e] = stack.pop()
    slots = []
    for b, (k, n, u) in enumerate(zip(keep, lens, used)):
        for i in range(n):
            at = k + i
            slots.append(new[b][at // page] * page + at % page if i < u else -1)
    slots = (slots + [-1] * rows_ub)[:rows_ub]
    return dict(table=new, free=stack, kv_len=[k + u for k, u in zip(keep, used)], slots=slots, status=0)


def cached_rows(pool_k, pool_v, table_row, n):
    """The first n tokens of a request: k, v [n, kv, dim] and whether each one's
    page is one of the pool (zeros where not).  pool_*: [pages, kv, page, dim]."""
    P, KV, page, D = pool_k.shape
    k, v, ok = np.zeros((n, KV, D)), np.zeros((n, KV, D)), np.zeros(n, bool)
    for t in range(n):
        p = int(table_row[t // page])
        if 0 <= p < P:
            k[t], v[t], ok[t] = pool_k[p, :, t % page], pool_v[p, :, t % page], True
    return k, v, ok


def sees(mask, n_rows, n_keys, bits=None):
    """[n_rows, n_keys] bool; the rows are the last n_rows of the n_keys
    positions.  mask: "none" | "causal" | "tree"; bits: [n_rows] Python ints."""
    past = n_keys - n_rows
    out = np.ones((n_rows, n_keys), bool)
    for i in range(n_rows):
        for j in range(n_keys):
            if mask == "causal":
                out[i, j] = j <= past + i
            elif mask == "tree" and j >= past:
                out[i, j] = bits[i] >> (j - past) & 1
    return out


def attend(q, k, v, seen, scale=None):
    """q [n, H, D], k, v [L, KV, D], seen [n, L] -> (o [n, H, D], sum_j p_j |v_j|
    of the same shape, largest scale * sum_d |q_d k_jd| of each row and head
    [n, H]): the second and third are what an error bound needs."""
    n, H, D = q.shape
    G = H // k.shape[1]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    o, absum, mag = np.zeros((n, H, D)), np.zeros((n, H, D)), np.zeros((n, H))
    for i in range(n):
        at = np.nonzero(seen[i])[0]
        if at.size == 0:
            continue
        for h in range(H):
            kk, vv = k[at, h // G], v[at, h // G]
            with np.errstate(invalid="ignore"):          # infinities of opposite signs among what the row sees
                s = scale * (kk @ q[i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                o[i, h], absum[i, h] = p @ vv, p @ np.abs(vv)
                mag[i, h] = abs(scale) * (np.abs(kk) @ np.abs(q[i, h])).max()
    return o, absum, mag
