"""Sequencing of the C-ABI calls for the whole Seer path on one GPU.

Device memory comes from torch (plumbing only); every step of the path --
layer forwards, the fused near-zero count, the SNR scan, routing and
compaction -- is one of libseer's entry points.  The step-0 pipeline follows
the method's order (Sec. 3.2-3.5): layers 0..l_det on the full window with
the count at l_det, boundary detection, route + compaction of the in-flight
residual and of the step-input embeddings in one launch, then the remaining
layers on the compacted batch.  Later denoising steps run every layer on the
compacted batch, or, with the prefix keys/values cached (Appendix D), on the
kept window rows alone.

Graph-compatible execution (Sec. 3.5): every kernel reads its row counts from
device memory, so one recorded launch sequence (a HIP graph, recorded through
the library's seer_graph_* calls) serves any batch whose routed capacity fits
the rows bound it was recorded with.  The repack kernel writes the routed
shape to pinned host memory; the host polls that word, without waiting on the
stream, to pick the recorded sequence for the capacity.
"""
import time
from dataclasses import dataclass
from typing import Dict, List, Optional

import torch

from . import seer as S


def dims_for(d_model, n_heads, head_dim, d_ff, dtype, rms_eps=1e-5, rope_theta=0.0):
    return S.seer_dims(d_model, n_heads, head_dim, d_ff,
                       S.SEER_DTYPE_BF16 if dtype == "bf16" else S.SEER_DTYPE_F32, rms_eps, rope_theta)


def torch_dtype(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


CTRL_FIELDS = ("total_rows", "capacity_rows", "n_static", "n_varlen", "n_eager", "n_groups", "max_alloc",
               "status", "ready")


def pinned_ctrl():
    """A host-pinned control word (16 int32) for seer_batch_repack."""
    return torch.zeros(16, dtype=torch.int32, pin_memory=True)


def poll_ctrl(ctrl_host, timeout_s=30.0):
    """Spin on the pinned control word until the repack kernel has written it
    (its ready field is stored last), without synchronising any stream.
    Returns the fields as a dict.  The caller clears `ready` (ctrl_host[8] = 0)
    before enqueuing the repack."""
    a = ctrl_host.numpy()
    t_end = time.monotonic() + timeout_s
    spins = 0
    while int(a[8]) != 1:
        spins += 1
        if spins > 1000:
            time.sleep(5e-5)           # past the first ~100 us, yield the core between reads
        if time.monotonic() > t_end:
            raise TimeoutError("control word not written within %.0f s" % timeout_s)
    v = [int(a[i]) for i in range(9)]
    return dict(zip(CTRL_FIELDS, v))


def graph_shape(rows, granule=256):
    """The 1-D graph shape for a routed capacity: the smallest of granule x
    {1, 2, 3, 4, 6, 8, 12, 16, ...} (at most 1.5x over) that holds `rows`."""
    units = max(1, -(-int(rows) // granule))
    u = 1
    while u < units:
        if u >= 2 and u & (u - 1) == 0:
            u += u // 2            # 2^k -> 1.5 x 2^k
        elif u % 3 == 0:
            u = u // 3 * 4         # 1.5 x 2^k -> 2^(k+1)
        else:
            u = 2 * u
    return u * granule


class SeerGraph:
    """A recorded launch sequence; replay() runs it on a stream."""

    def __init__(self, handle):
        self.handle = handle

    def replay(self, stream=None):
        S.seer_graph_launch(self.handle, stream=stream)

    def close(self):
        if self.handle:
            S.seer_graph_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def record(fn, stream):
    """Record the seer calls fn() issues on `stream` (a created torch stream;
    fn must issue nothing else on it) into a SeerGraph."""
    S.seer_graph_begin(stream)
    try:
        fn()
    except BaseException:
        # close the recording, drop what it holds, and report fn's error
        try:
            S.seer_graph_destroy(S.seer_graph_end(stream))
        except S.SeerError:
            pass
        raise
    return SeerGraph(S.seer_graph_end(stream))


@dataclass
class Step0Result:
    counts: torch.Tensor        # [rows_full] int32 at the detection layer
    boundary: torch.Tensor      # [B] int32
    keep_len: torch.Tensor      # [B] int32
    cu_trunc: torch.Tensor      # [B+1] int32
    seqused: torch.Tensor       # [B] int32
    route: torch.Tensor         # [B, 3] int32
    ctrl: torch.Tensor          # [16] int32 (device copy of the control word)
    x_trunc: torch.Tensor       # compacted step-input embeddings
    h_trunc: torch.Tensor       # step-0 residual after the last layer (compacted)
    routed: Optional[dict] = None   # the control word read from pinned memory (if polled)
    rows_ub: int = 0            # rows bound the layers after the repack ran with


class StepGraphs:
    """Recorded denoising steps, one per 1-D graph shape (Sec. 3.5).

    step_fn(rows_ub) issues one step's seer calls on `stream`, on buffers that
    stay fixed for the life of this object; run(capacity_rows) replays the
    recording for graph_shape(capacity_rows) (recorded on first use)."""

    def __init__(self, step_fn, stream, max_rows, granule=256):
        self.step_fn = step_fn
        self.stream = stream
        self.max_rows = int(max_rows)
        self.granule = granule
        self.graphs: Dict[int, SeerGraph] = {}

    def shape(self, capacity_rows):
        return min(graph_shape(capacity_rows, self.granule), self.max_rows)

    def run(self, capacity_rows):
        rows = self.shape(capacity_rows)
        g = self.graphs.get(rows)
        if g is None:
            g = record(lambda: self.step_fn(rows), self.stream)
            self.graphs[rows] = g
        g.replay(self.stream)
        return rows

    def close(self):
        for g in self.graphs.values():
            g.close()
        self.graphs.clear()


class SyntheticSampler:
    """LM head and low-confidence remasking between denoising steps, on
    window-only rows (the layout of the cached-prefix steps): after a step,
    every masked window position gets a prediction and a confidence, the most
    confident are committed, and the next step's input rows are rebuilt from
    the committed tokens' embeddings (uncommitted rows keep their step-0
    input).  Token state: tokens[r] == -1 while masked."""

    def __init__(self, dims, w_lm, emb, rows_ub, device="cuda"):
        self.dims = dims
        self.emb = emb
        self.vocab = int(w_lm.shape[0])
        self.rows_ub = int(rows_ub)
        # the head weight in the matrix cores' operand order (the row-major
        # w_lm is not kept)
        self.w_packed = torch.empty(w_lm.numel() * 2, dtype=torch.uint8, device=device)
        S.seer_lm_head_prepack(dims, w_lm, self.vocab, self.w_packed)
        torch.cuda.current_stream(self.w_packed.device).synchronize()   # later calls may use other streams
        self.ws_bytes = S.seer_lm_head_workspace_bytes(dims, self.vocab, self.rows_ub)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self.pred = torch.empty(self.rows_ub, dtype=torch.int32, device=device)
        self.conf = torch.empty(self.rows_ub, dtype=torch.float32, device=device)
        self.tokens = torch.full((self.rows_ub,), -1, dtype=torch.int32, device=device)

    def reset(self):
        self.tokens.fill_(-1)

    def predict(self, h, cu, batch, rows_ub, stream=None):
        S.seer_lm_head_predict(self.dims, self.w_packed, self.vocab, h, rows_ub, cu, batch, self.pred, self.conf,
                               self.workspace, self.ws_bytes, stream=stream)

    def step(self, h, cu, used, batch, rows_ub, x0, x_next, steps_left, max_used, stream=None):
        """Predict on the step's output rows h, commit, write the next inputs."""
        self.predict(h, cu, batch, rows_ub, stream=stream)
        S.seer_remask_step(self.dims, cu, used, batch, max_used, steps_left, self.pred, self.conf, self.tokens,
                           x0, self.emb, self.vocab, x_next, stream=stream)


class PagedCache:
    """Keys and values of up to max_batch requests in pages, one pool per layer
    with one table for all: what seer_page_plan, seer_kv_store, seer_attn_paged
    and seer_attn_prompt work on.  A step of a program is

        slots = cache.plan(cu, rows_ub, keep)      # pages taken and given back
        for each layer:
            cache.store(layer, k, v, rows_ub, slots)
            cache.attend(layer, q, out, cu, rows_ub, mask)

    with the rows of request b at [cu[b], cu[b+1]) (none for a place that is
    not in use).  keep[b]: tokens of the request that stay from earlier steps
    (None: all), fewer where a window was cut or drafts were refused, 0 where
    the request has ended.  Lengths and free pages stay on the device; each plan
    reads one of two buffers and writes the other, so a recorded sequence has an
    even number of plans.  The calls go to the current stream (or `stream`) of
    the cache's device, which has to be the current one; they share a workspace,
    so that calls on two streams, recordings among them, may not overlap.

    Rows of q, k, v and out are [at least rows_ub, heads * head_dim], or more dims
    with the same elements, in the cache's types, a row's side by side in memory
    (row strides are free), tree_bits [at least rows_ub, words] int64 and contiguous,
    cu, keep, seqused and slots int32 and contiguous; ValueError otherwise."""

    _invalid = "keep exceeds what a request holds"

    def __init__(self, n_heads, n_kv_heads, head_dim, n_layers, n_pages, page_size, max_batch, max_len, max_rows,
                 dtype="bf16", v_f16=False, scale=0.0, device="cuda"):
        S.load_library()
        self.desc = S.seer_attn_desc(n_heads, n_kv_heads, head_dim,
                                     S.SEER_DTYPE_BF16 if dtype == "bf16" else S.SEER_DTYPE_F32,
                                     S.SEER_ATTN_V_F16 if v_f16 else 0, scale)
        width = -(-int(max_len) // int(page_size))
        self.pages = S.seer_page_desc(page_size, n_pages, width)
        nbytes = S.seer_page_pool_bytes(self.desc, self.pages)
        self.ws_bytes = S.seer_attn_workspace_bytes(self.desc, max_rows, max_batch)
        if nbytes == 0 or self.ws_bytes == 0:
            raise S.SeerError(S.SEER_EUNSUPPORTED, S.seer_last_error())
        self.max_batch, self.max_rows = int(max_batch), int(max_rows)
        kind = torch_dtype(dtype)
        self.kind, self.v_kind = kind, torch.float16 if v_f16 else kind
        self.q_width, self.kv_width = n_heads * head_dim, n_kv_heads * head_dim
        shape = (n_pages, 2, n_kv_heads, page_size, head_dim)
        self.pools = [torch.zeros(shape, dtype=kind, device=device) for _ in range(n_layers)]
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)
        self.table = i32(max_batch, width)
        # page 0 is the first one taken
        self.free_pages = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        self._free = [torch.full((1,), n_pages, dtype=torch.int32, device=device), i32(1)]
        self._lens = [i32(max_batch), i32(max_batch)]
        self.slots = i32(max_rows)
        self._planned = 0                             # rows whose slots are the last plan's
        self.status = i32(1)
        self.refused = i32(1)                         # the bits of every refused plan since the last check
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        self._device = self.table.get_device()        # -1 on the CPU

    @property
    def lens(self):
        """[max_batch] int32: the tokens that each request has in the cache."""
        return self._lens[0]

    @property
    def free(self):
        """[1] int32: the number of free pages."""
        return self._free[0]

    def _takes(self, rows_ub, cu=None, keep=None, seqused=None, slots=None):
        """Refuse what the kernels would read or write past an end, or misread."""
        if self._device >= 0 and torch.cuda.current_device() != self._device:
            raise ValueError("the cache is on %s, which is not the current device" % (self.table.device,))
        if rows_ub > self.max_rows:
            raise ValueError("rows_ub %d exceeds max_rows %d" % (rows_ub, self.max_rows))
        if cu is not None:
            self._ints("cu", cu, self.max_batch + 1)
        if keep is not None:
            self._ints("keep", keep, self.max_batch)
        if seqused is not None:
            self._ints("seqused", seqused, self.max_batch)
        if slots is not None:
            self._ints("slots", slots, rows_ub)

    def _slots(self, rows_ub, slots):
        """The slots of a store; of the cache's own, no more than the last plan wrote."""
        if slots is None or slots is self.slots:
            if rows_ub > self._planned:
                raise ValueError("rows_ub %d exceeds the %d rows of the last plan" % (rows_ub, self._planned))
            return self.slots
        return slots

    def _ints(self, name, x, n):
        if x.numel() < n:
            raise ValueError("%s has %d entries, %d needed" % (name, x.numel(), n))
        if x.dtype is not torch.int32 or not x.is_contiguous() or x.get_device() != self._device:
            raise ValueError("%s has to be int32, contiguous and on the cache's device" % name)

    def _rows(self, rows_ub, name, x, width, kind):
        """The same for rows of q, k, v and the output."""
        if x.dtype is not kind or x.get_device() != self._device:
            raise ValueError("%s has to be %s on the cache's device" % (name, kind))
        shape, stride = x.shape, x.stride()
        n = shape[1] if len(shape) == 2 and stride[1] == 1 else self._side_by_side(shape, stride)
        if n < width:
            raise ValueError("%s has to have rows of %d elements side by side" % (name, width))
        if shape[0] < rows_ub:
            raise ValueError("%s has %d rows, fewer than rows_ub %d" % (name, shape[0], rows_ub))

    def _bits(self, rows_ub, tree_bits):
        if tree_bits is not None:
            if tree_bits.dtype not in (torch.int64, torch.uint64) or tree_bits.get_device() != self._device or \
                    tree_bits.dim() != 2 or not tree_bits.is_contiguous() or tree_bits.shape[0] < rows_ub:
                raise ValueError("tree_bits has to be [at least %d, words] int64, contiguous and on the cache's device"
                                 % rows_ub)

    @staticmethod
    def _side_by_side(shape, stride):
        """Elements of a row that lie one after the other in memory, 0 where it has gaps."""
        n = 1 if len(shape) > 1 else 0
        for size, step in zip(shape[:0:-1], stride[:0:-1]):
            if size != 1 and step != n:
                return 0
            n *= size
        return n

    def plan(self, cu, rows_ub, keep=None, seqused=None, stream=None):
        """The pages and slots of a step; returns the slots of its rows."""
        return self._plan(cu, rows_ub, keep, seqused, stream)

    def _plan(self, cu, rows_ub, keep, seqused, stream, kept=None):
        self._takes(rows_ub, cu, keep, seqused)
        held = self._lens[0]
        S.seer_page_plan_latched(self.pages, held, held if keep is None else keep, cu, seqused, self.max_batch, rows_ub,
                                 self.free_pages, self._free[0], self._free[1], self.table, self._lens[1], self.slots,
                                 self.status, self.refused, stream=stream, kept=kept)
        self._lens.reverse()
        self._free.reverse()
        self._planned = rows_ub
        return self.slots

    def check(self, stream=None):
        """Raise SeerError if a plan since the last check was refused, in a recording too; waits for `stream`."""
        if stream is None:
            stream = torch.cuda.current_stream(self.status.device)
        elif isinstance(stream, int):                 # a raw handle, as the other calls take it
            stream = torch.cuda.ExternalStream(stream, self.status.device) if stream else \
                torch.cuda.default_stream(self.status.device)
        stream.synchronize()
        st = int(self.refused.item())
        if st:
            self.refused.zero_()
            if self._device >= 0:
                torch.cuda.current_stream(self.status.device).synchronize()     # before plans on other streams
            why = [n for bit, n in ((S.SEER_PAGES_EXHAUSTED, "not enough free pages"),
                                    (S.SEER_PAGES_WIDTH, "a request longer than max_len"),
                                    (S.SEER_PAGES_INVALID, self._invalid)) if st & bit]
            raise S.SeerError(S.SEER_EWORKSPACE, "; ".join(why))

    def store(self, layer, k, v, rows_ub, slots=None, stream=None):
        """Rows of k and v ([rows, n_kv_heads * head_dim], any row stride) into the layer's pages."""
        self._takes(rows_ub, slots=slots)
        self._rows(rows_ub, "k", k, self.kv_width, self.kind)
        self._rows(rows_ub, "v", v, self.kv_width, self.v_kind)
        S.seer_kv_store(self.desc, self.pages, k, k.stride(0), v, v.stride(0), rows_ub, self._slots(rows_ub, slots),
                        self.pools[layer], stream=stream)

    def store_layer(self, layer, stack, rows_ub, slots=None, stream=None):
        """The K | V columns that the stack's last layer call left in its
        workspace (made with the same rows_ub) into the layer's pages: the paged
        counterpart of seer_kv_export.  A bf16 layer leaves V in fp16, so the
        cache has to have v_f16."""
        k, d, es = self._layer_rows(layer, stack, rows_ub, slots)
        S.seer_kv_store(self.desc, self.pages, k, 3 * d, k + d * es, 3 * d, rows_ub,
                        self._slots(rows_ub, slots), self.pools[layer], stream=stream)

    def _layer_rows(self, layer, stack, rows_ub, slots):
        """(address of the K columns in the stack's workspace, their number, bytes of an element)."""
        d, bf16 = stack.dims.d_model, stack.dtype == torch.bfloat16
        flags = S.SEER_ATTN_V_F16 if bf16 else 0
        if (self.desc.n_kv_heads * self.desc.head_dim, self.desc.dtype, self.desc.flags) != (d, stack.dims.dtype, flags):
            raise ValueError("the cache's heads and types are not those of the layer's rows")
        self._takes(rows_ub, slots=slots)
        es = 2 if bf16 else 4
        return stack.workspace.data_ptr() + S.seer_layer_workspace_offsets(stack.dims, rows_ub)[0] + d * es, d, es

    def attend(self, layer, q, out, cu, rows_ub, mask=S.SEER_MASK_CAUSAL, tree_bits=None, seqused=None, stream=None):
        """Attention of the step's rows over their requests' pages."""
        self._takes(rows_ub, cu, None, seqused)
        self._rows(rows_ub, "q", q, self.q_width, self.kind)
        self._rows(rows_ub, "out", out, self.q_width, self.kind)
        self._bits(rows_ub, tree_bits)
        S.seer_attn_paged(self.desc, self.pages, mask, q, q.stride(0), out, out.stride(0), rows_ub, cu, seqused,
                          self.max_batch, self.pools[layer], self.table, self._lens[0], tree_bits,
                          0 if tree_bits is None else tree_bits.shape[1], self.workspace, self.ws_bytes, stream=stream)

    def prompt(self, q, k, v, out, cu, rows_ub, mask=S.SEER_MASK_CAUSAL, seqused=None, stream=None):
        """Attention of packed prompts over their own rows (no pages)."""
        self._takes(rows_ub, cu, None, seqused)
        self._rows(rows_ub, "q", q, self.q_width, self.kind)
        self._rows(rows_ub, "k", k, self.kv_width, self.kind)
        self._rows(rows_ub, "v", v, self.kv_width, self.v_kind)
        self._rows(rows_ub, "out", out, self.q_width, self.kind)
        S.seer_attn_prompt(self.desc, mask, q, q.stride(0), k, k.stride(0), v, v.stride(0), out, out.stride(0),
                           rows_ub, cu, seqused, self.max_batch, self.workspace, self.ws_bytes, stream=stream)


class BudgetCache(PagedCache):
    """A PagedCache that stays within a budget: keys carry rotary positions, every
    token the attention weight that it has had, and evict() keeps the heaviest
    (seer_kv_store_rope, seer_row_positions, seer_attn_weights, seer_kv_evict).
    A step of a program is

        cache.plan(cu, rows_ub)                    # pages, slots, positions
        for each layer:
            cache.store(layer, k, v, rows_ub, q=q)            # q and k rotated
            cache.attend(layer, q, out, cu, rows_ub, mask)
            cache.weigh(layer, q, cu, rows_ub, mask)
        for each layer:                            # now and then
            cache.evict(layer, budget)             # the next plan gives the pages back

    rope: a seer_rope_desc, or None for keys that are stored as they are.  seen
    counts the tokens that each request has had; plan() goes on from it, or from
    `base` where drafts were refused (with the `keep` that goes with them) or a
    request has ended (0).  After evict() has cut every layer alike, plan() keeps
    what it kept; a `keep` of the caller's may keep less, and one that keeps more is
    refused.  A cut layer takes no other call before that plan, and no plan comes
    between the layers of one cut: ValueError.  Where layers were cut to different
    lengths that plan is refused; a `keep` up to the least of them is taken then.
    Calls after a refused plan mean nothing until check() has raised it: nothing is
    stored or cut, and what was cut before stays so (weigh() adds to the weights).

    What stays of each request is counted on the device (kept: the tokens after
    the last plan, or what evict() has left of them), so that a recording may
    begin and end before a cut or behind one, and be replayed among eager steps.
    The ValueErrors go by the order in which calls are made, and a recorded call
    is made when it is recorded: behind a recording that ends with a cut, eager
    calls go on with plan().

    rows, types and streams as for PagedCache; budget, base int32 [max_batch]."""

    _invalid = "keep exceeds what a request holds, or its layers were cut to different lengths"

    def __init__(self, n_heads, n_kv_heads, head_dim, n_layers, n_pages, page_size, max_batch, max_len, max_rows,
                 rope=None, dtype="bf16", v_f16=False, scale=0.0, device="cuda"):
        super().__init__(n_heads, n_kv_heads, head_dim, n_layers, n_pages, page_size, max_batch, max_len, max_rows,
                         dtype=dtype, v_f16=v_f16, scale=scale, device=device)
        self.rope, self.turns = rope, None
        if rope is not None:
            self.turns = torch.tensor(S.seer_rope_turns(rope, head_dim), dtype=torch.float64, device=device)
        marks = (n_pages, n_kv_heads, page_size)
        self.weights = [torch.zeros(marks, dtype=torch.float32, device=device) for _ in range(n_layers)]
        self.numbers = [torch.zeros(marks, dtype=torch.int32, device=device) for _ in range(n_layers)]
        self._seen = [torch.zeros(max_batch, dtype=torch.int32, device=device) for _ in range(2)]
        self.positions = torch.zeros(max_rows, dtype=torch.int32, device=device)
        self.kept = torch.zeros(max_batch, dtype=torch.int32, device=device)      # what the next plan keeps
        self._cut = set()                             # layers that are cut since the last plan
        self._cut_before = set()                      # and before it
        need = max(S.seer_attn_weights_workspace_bytes(self.desc, self.pages, max_rows, max_batch),
                   S.seer_kv_evict_workspace_bytes(self.desc, self.pages, max_batch), self.ws_bytes)
        if need > self.ws_bytes:
            self.ws_bytes = need
            self.workspace = torch.empty(need, dtype=torch.uint8, device=device)

    @property
    def seen(self):
        """[max_batch] int32: the tokens that each request has had, the position of its next."""
        return self._seen[0]

    def _whole(self, layer):
        if layer in self._cut:
            raise ValueError("layer %d is cut: the next call is plan()" % layer)

    @staticmethod
    def _apart(name, x, *written):
        """Refuse an argument that shares memory with what the same call writes."""
        a = x.data_ptr()
        end = a + x.numel() * x.element_size()
        for w in written:
            b = w.data_ptr()
            if a < b + 4 * w.numel() and b < end:
                raise ValueError("%s may not be in a buffer that the call writes" % name)

    def plan(self, cu, rows_ub, keep=None, seqused=None, base=None, stream=None):
        """The pages, slots and positions of a step; returns the slots of its rows."""
        if base is not None:
            self._ints("base", base, self.max_batch)
        # (before the pages are planned: the positions come behind them)
        for name, x in (("cu", cu), ("seqused", seqused), ("base", base)):
            if x is not None:
                self._apart(name, x, self.kept, self._seen[1])
        if self._cut:
            if len(self._cut) < len(self.pools):
                raise ValueError("%d of %d layers are cut: a plan comes after all or none" % (len(self._cut), len(self.pools)))
        slots = self._plan(cu, rows_ub, self.kept if keep is None else keep, seqused, stream, self.kept)
        self._cut_before, self._cut = self._cut, set()
        S.seer_row_positions(cu, seqused, self.max_batch, self._seen[0], base, self.status, rows_ub, self.positions,
                             self._seen[1], stream=stream, kv_len=self._lens[0], kept=self.kept)
        self._seen.reverse()
        return slots

    def check(self, stream=None):
        """As PagedCache.check; where the last plan was refused, what was cut before it still is."""
        try:
            super().check(stream)
        except S.SeerError:
            self._cut |= self._cut_before
            raise

    def _positions(self, rows_ub, positions):
        if positions is None or positions is self.positions:
            if rows_ub > self._planned:
                raise ValueError("rows_ub %d exceeds the %d rows of the last plan" % (rows_ub, self._planned))
            return self.positions
        self._ints("positions", positions, rows_ub)
        return positions

    def rotate(self, q, k, rows_ub, q_out=None, k_out=None, positions=None, inverse=False, stream=None):
        """Rotary positions of rows of q and k (None: not these), in place or to q_out and k_out: for prompt()."""
        self._takes(rows_ub)
        positions = self._positions(rows_ub, positions)
        q_out, k_out = q if q_out is None else q_out, k if k_out is None else k_out
        for name, x, width in (("q", q, self.q_width), ("q_out", q_out, self.q_width), ("k", k, self.kv_width),
                               ("k_out", k_out, self.kv_width)):
            if x is not None:
                self._rows(rows_ub, name, x, width, self.kind)
        row = lambda x: 0 if x is None else x.stride(0)
        S.seer_rope_rows(self.desc, self.rope, self.turns, S.SEER_ROPE_INVERSE if inverse else 0, q, row(q), k, row(k),
                         q_out, row(q_out), k_out, row(k_out), rows_ub, positions, stream=stream)

    def store(self, layer, k, v, rows_ub, slots=None, stream=None, q=None, q_out=None, positions=None):
        """Rows of k, rotated, and v into the layer's pages, with new marks; q, if given, rotated in place or to q_out."""
        self._takes(rows_ub, slots=slots)
        self._whole(layer)
        self._rows(rows_ub, "k", k, self.kv_width, self.kind)
        self._rows(rows_ub, "v", v, self.kv_width, self.v_kind)
        q_out = q if q_out is None else q_out
        for name, x in (("q", q), ("q_out", q_out)):
            if x is not None:
                self._rows(rows_ub, name, x, self.q_width, self.kind)
        row = lambda x: 0 if x is None else x.stride(0)
        S.seer_kv_store_rope(self.desc, self.pages, self.rope, self.turns, q, row(q), q_out, row(q_out), k, k.stride(0),
                             v, v.stride(0), rows_ub, self._positions(rows_ub, positions), self._slots(rows_ub, slots),
                             self.pools[layer], self.weights[layer], self.numbers[layer], stream=stream)

    def store_layer(self, layer, stack, rows_ub, slots=None, stream=None):
        """As PagedCache.store_layer, with new marks: the layer's keys carry its own positions and are not rotated again."""
        self._whole(layer)
        k, d, es = self._layer_rows(layer, stack, rows_ub, slots)
        S.seer_kv_store_rope(self.desc, self.pages, None, None, None, 0, None, 0, k, 3 * d, k + d * es, 3 * d, rows_ub,
                             self._positions(rows_ub, None), self._slots(rows_ub, slots), self.pools[layer],
                             self.weights[layer], self.numbers[layer], stream=stream)

    def attend(self, layer, q, out, cu, rows_ub, mask=S.SEER_MASK_CAUSAL, tree_bits=None, seqused=None, stream=None):
        """Attention of the step's rows over their requests' pages."""
        self._whole(layer)
        super().attend(layer, q, out, cu, rows_ub, mask, tree_bits, seqused, stream=stream)

    def weigh(self, layer, q, cu, rows_ub, mask=S.SEER_MASK_CAUSAL, tree_bits=None, seqused=None, last=0, decay=1.0,
              stream=None):
        """Add the attention weight that the step's rows (of each request the last `last`, 0: all) give to the
        cached tokens, whose weights so far count `decay` times."""
        self._takes(rows_ub, cu, None, seqused)
        self._whole(layer)
        self._rows(rows_ub, "q", q, self.q_width, self.kind)
        self._bits(rows_ub, tree_bits)
        w = self.weights[layer]
        S.seer_attn_weights(self.desc, self.pages, mask, q, q.stride(0), rows_ub, cu, seqused, self.max_batch, last,
                            self.pools[layer], self.table, self._lens[0], tree_bits,
                            0 if tree_bits is None else tree_bits.shape[1], decay, w, w, self.workspace, self.ws_bytes,
                            stream=stream)

    def evict(self, layer, budget, first=0, recent=0, shared=False, stream=None):
        """Cut each request's cache in this layer to budget[b] tokens; returns the lengths kept (-1 - the least of them
        where layers were cut to different ones).  Takes effect with the next plan, and all layers are cut alike before it."""
        self._takes(0)
        self._whole(layer)
        self._ints("budget", budget, self.max_batch)
        if budget.data_ptr() != self.kept.data_ptr():
            self._apart("budget", budget, self.kept)
        w, n = self.weights[layer], self.numbers[layer]
        flags = (S.SEER_EVICT_SHARED if shared else 0) | (S.SEER_EVICT_ALIKE if self._cut else 0)
        S.seer_kv_evict(self.desc, self.pages, flags, self._lens[0], budget, self._seen[0],
                        self.max_batch, first, recent, self.table, self.pools[layer], w, n, w, n, self.kept,
                        self.workspace, self.ws_bytes, stream=stream, status=self.status)
        self._cut.add(layer)
        return self.kept


class SeerStack:
    """A stack of prepacked layers plus the scratch the ABI calls need."""

    def __init__(self, dims, n_layers, max_rows, device="cuda"):
        S.load_library()
        self.dims = dims
        self.n_layers = n_layers
        self.max_rows = int(max_rows)
        self.device = device
        self.dtype = torch.bfloat16 if dims.dtype == S.SEER_DTYPE_BF16 else torch.float32
        self.packed_bytes = S.seer_prepacked_bytes(dims)
        if self.packed_bytes == 0:
            raise S.SeerError(S.SEER_EUNSUPPORTED, S.seer_last_error())
        self.packed: List[Optional[torch.Tensor]] = [None] * n_layers
        self.ws_bytes = S.seer_layer_workspace_bytes(dims, self.max_rows)
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        S.seer_layer_status_reset(self.workspace, self.ws_bytes)
        d = dims.d_model
        self.buf = [torch.zeros(self.max_rows, d, dtype=self.dtype, device=device) for _ in range(2)]
        self._trunc_bufs = {}

    def layer_status(self, stream=None):
        """The workspace status word (SEER_STATUS_* bits accumulated by every
        layer call since construction or the last reset); waits for `stream`."""
        (stream or torch.cuda.current_stream(self.workspace.device)).synchronize()
        return int(self.workspace[:4].view(torch.int32).item())

    def check_status(self, stream=None):
        """Raise SeerError if a layer call reported a value out of range."""
        st = self.layer_status(stream)
        if st & S.SEER_STATUS_V_RANGE:
            raise S.SeerError(S.SEER_EUNSUPPORTED, "an attention value exceeded the fp16 range (|v| > 65504)")

    def reset_status(self, stream=None):
        S.seer_layer_status_reset(self.workspace, self.ws_bytes, stream=stream)

    def set_layer(self, l, weights, stream=None):
        if self.packed[l] is None:
            self.packed[l] = torch.empty(self.packed_bytes, dtype=torch.uint8, device=self.device)
        S.seer_prepack_weights(self.dims, weights, self.packed[l], stream=stream)

    def layer(self, l, x_in, x_out, cu, seqused, batch, rows_ub, act_eps=0.0, act_count=None,
              stream=None):
        S.seer_layer_forward_varlen(self.dims, self.packed[l], x_in, x_out, rows_ub, cu, seqused,
                                    batch, act_eps, act_count, self.workspace, self.ws_bytes,
                                    stream=stream)

    def forward(self, x, cu, seqused, batch, rows_ub, layers=None, out=None, stream=None):
        """Run layers (default all) over x; returns the output tensor."""
        layers = range(self.n_layers) if layers is None else layers
        cur = x
        for i, l in enumerate(layers):
            nxt = self.buf[i % 2] if cur is not self.buf[i % 2] else self.buf[(i + 1) % 2]
            self.layer(l, cur, nxt, cu, seqused, batch, rows_ub, stream=stream)
            cur = nxt
        if out is not None and cur is not out:
            out[:rows_ub].copy_(cur[:rows_ub])
            cur = out
        return cur

    # ---- truncated steps with the prefix keys/values cached (Appendix D) ----
    def alloc_kv_caches(self, kv_rows):
        """One [kv_rows, 2 d] cache per layer (K | V, the qkv element types)."""
        return [torch.empty(max(int(kv_rows), 1), 2 * self.dims.d_model, dtype=self.dtype,
                            device=self.device) for _ in range(self.n_layers)]

    def forward_export(self, x, cu, seqused, batch, rows_ub, caches, cu_kv, kv_rows_ub, out=None,
                       stream=None):
        """A full truncated step over [prefix; kept window] rows that also
        caches, per layer, the K | V of each sequence's first cu_kv[b+1] - cu_kv[b]
        rows."""
        cur = x
        for l in range(self.n_layers):
            nxt = self.buf[l % 2] if cur is not self.buf[l % 2] else self.buf[(l + 1) % 2]
            self.layer(l, cur, nxt, cu, seqused, batch, rows_ub, stream=stream)
            S.seer_kv_export(self.dims, self.workspace, rows_ub, cu, batch, cu_kv, kv_rows_ub, caches[l],
                             workspace_bytes=self.ws_bytes, stream=stream)
            cur = nxt
        if out is not None and cur is not out:
            out[:rows_ub].copy_(cur[:rows_ub])
            cur = out
        return cur

    def forward_cached(self, x_w, cu_w, used_w, batch, rows_ub, caches, cu_kv, kv_rows_ub, out=None,
                       stream=None):
        """A truncated step on the kept window rows only, every layer reading
        its cached prefix keys/values."""
        cur = x_w
        for l in range(self.n_layers):
            nxt = self.buf[l % 2] if cur is not self.buf[l % 2] else self.buf[(l + 1) % 2]
            S.seer_layer_forward_cached(self.dims, self.packed[l], cur, nxt, rows_ub, cu_w, used_w, batch,
                                        caches[l], cu_kv, kv_rows_ub, self.workspace, self.ws_bytes,
                                        stream=stream)
            cur = nxt
        if out is not None and cur is not out:
            out[:rows_ub].copy_(cur[:rows_ub])
            cur = out
        return cur

    def window_rows(self, src, cu_src, win_off, win_len, keep, batch, capacity, policy=S.SEER_ROUTE_HYBRID,
                    tau_pad=(1, 5), granule=256, ctrl_host=None, stream=None):
        """The kept window rows of each sequence of `src`, routed and compacted
        (no prefix rows): returns (rows, cu, seqused, route).  The buffers are
        owned by the stack and reused by the next call of the same shape.  With
        ctrl_host (pinned_ctrl()), the routed shape is also written there for
        poll_ctrl; its ready field is cleared here before the launch."""
        dev = self.device
        key = ("win", capacity, batch)
        if key not in self._trunc_bufs:
            self._trunc_bufs[key] = (
                torch.empty(capacity, self.dims.d_model, dtype=self.dtype, device=dev),
                torch.empty(batch + 1, dtype=torch.int32, device=dev),
                torch.empty(batch, dtype=torch.int32, device=dev),
                torch.empty(batch, 3, dtype=torch.int32, device=dev))
        dst, cu, used, route = self._trunc_bufs[key]
        desc = S.seer_repack_desc(policy, tau_pad[0], tau_pad[1], granule,
                                  self.dims.d_model * (2 if self.dtype == torch.bfloat16 else 4),
                                  capacity, 0, S.SEER_REPACK_WINDOW_ONLY)
        if ctrl_host is not None:
            ctrl_host[8] = 0
        S.seer_batch_repack(desc, [src], [dst], cu_src, win_off, win_len, keep, batch, cu, used, route,
                            ctrl_host=ctrl_host, stream=stream)
        return dst, cu, used, route

    def step0(self, x_full, cu_full, win_off, win_len, batch, rows_full, l_det, act_eps,
              snr=(3, 100, 3, 5, 3), policy=S.SEER_ROUTE_HYBRID, tau_pad=(1, 5), granule=256,
              trunc_capacity=None, ctrl_host=None, check_status=True, stream=None):
        """Step 0 (Sec. 3.2-3.5): layers 0..l_det on the full window with the
        near-zero count at l_det and the SNR scan inside that layer (whose
        down projection then runs on the kept rows only), routing +
        compaction of the step-input embeddings and the in-flight residual,
        then the remaining layers on the compacted batch.

        trunc_capacity: rows of the compacted buffers.  By default the worst
        case of the routing: every window padded to the longest one,
        sum(win_off) + batch * max(win_len) rounded up to the granule (read
        from the device once).  A routed batch that does not fit is reported
        by the repack kernel in the control word; with ctrl_host it is read
        from the polled word, otherwise (check_status) from the device copy,
        and SeerError is raised before any later layer runs; that check also
        reads the workspace status word (check_status()).  The polled path
        never waits on the stream: its caller checks the status word when it
        syncs."""
        dev = self.device
        if trunc_capacity is None:
            wo = win_off[:batch].cpu().to(torch.int64)
            wl_ = win_len[:batch].cpu().to(torch.int64)
            worst = int(wo.sum()) + batch * int(wl_.max()) if batch > 0 else 0
            trunc_capacity = max(granule, -(-worst // granule) * granule)
        counts = torch.empty(rows_full, dtype=torch.int32, device=dev)
        cur = x_full
        for l in range(l_det):
            nxt = self.buf[l % 2]
            self.layer(l, cur, nxt, cu_full, None, batch, rows_full, stream=stream)
            cur = nxt
        cap = trunc_capacity
        key = (cap, batch)
        if key not in self._trunc_bufs:
            # compacted buffers, reused by every step0 call of this shape so that
            # recorded truncated steps keep valid addresses
            d = self.dims.d_model
            self._trunc_bufs[key] = dict(
                boundary=torch.empty(batch, dtype=torch.int32, device=dev),
                keep=torch.empty(batch, dtype=torch.int32, device=dev),
                x_t=torch.empty(cap, d, dtype=self.dtype, device=dev),
                h_t=torch.empty(cap, d, dtype=self.dtype, device=dev),
                cu_t=torch.empty(batch + 1, dtype=torch.int32, device=dev),
                used=torch.empty(batch, dtype=torch.int32, device=dev),
                route=torch.empty(batch, 3, dtype=torch.int32, device=dev),
                ctrl=torch.zeros(16, dtype=torch.int32, device=dev))
        tb = self._trunc_bufs[key]
        boundary, keep, x_t, h_t = tb["boundary"], tb["keep"], tb["x_t"], tb["h_t"]
        cu_t, used, route, ctrl = tb["cu_t"], tb["used"], tb["route"], tb["ctrl"]
        # the detection layer: count, scan, and its down projection on the kept rows only
        nxt = self.buf[l_det % 2]
        S.seer_layer_forward_detect(self.dims, self.packed[l_det], cur, nxt, rows_full, cu_full, batch, act_eps,
                                    counts, win_off, win_len, S.seer_snr_params(*snr), boundary, keep,
                                    self.workspace, self.ws_bytes, stream=stream)
        cur = nxt
        desc = S.seer_repack_desc(policy, tau_pad[0], tau_pad[1], granule,
                                  self.dims.d_model * (2 if self.dtype == torch.bfloat16 else 4),
                                  cap, 0, 0)
        if ctrl_host is not None:
            ctrl_host[8] = 0
        S.seer_batch_repack(desc, [x_full, cur], [x_t, h_t], cu_full, win_off, win_len, keep, batch,
                            cu_t, used, route, ctrl, ctrl_host, stream=stream)
        routed = None
        rows_ub = cap
        if ctrl_host is not None:
            # the routed capacity sizes the remaining launches (no stream sync)
            routed = poll_ctrl(ctrl_host)
            if routed["status"] != 0:
                raise S.SeerError(routed["status"], "compacted batch exceeds the %d-row buffers" % cap)
            rows_ub = max(1, min(cap, routed["capacity_rows"]))
        elif check_status:
            (stream or torch.cuda.current_stream(ctrl.device)).synchronize()   # the repack has written it
            status = int(ctrl[7].item())
            if status != 0:
                raise S.SeerError(status, "compacted batch exceeds the %d-row buffers" % cap)
            self.check_status(stream)           # the step-0 layers so far kept V in range
        if l_det + 1 < self.n_layers:
            h_t = self.forward(h_t, cu_t, used, batch, rows_ub, layers=range(l_det + 1, self.n_layers),
                               out=h_t, stream=stream)
        return Step0Result(counts=counts, boundary=boundary, keep_len=keep, cu_trunc=cu_t,
                           seqused=used, route=route, ctrl=ctrl, x_trunc=x_t, h_trunc=h_t,
                           routed=routed, rows_ub=rows_ub)
