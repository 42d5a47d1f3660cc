"""ctypes binding of libseer.so (include/seer.h), argument marshalling only.

Every function keeps the C name and argument order.  Pointer arguments accept
a torch tensor (its data_ptr), a plain integer address or None (NULL);
``stream`` defaults to torch's current HIP stream.  A non-zero status raises
SeerError carrying the library's message.  All arithmetic of the hot path
runs inside the library's HIP kernels; nothing here computes.
"""
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libseer.so")

SEER_OK, SEER_EINVAL, SEER_EUNSUPPORTED, SEER_EWORKSPACE, SEER_EHIP = 0, -1, -2, -3, -4
SEER_DTYPE_BF16, SEER_DTYPE_F32 = 1, 2
SEER_ROUTE_HYBRID, SEER_ROUTE_NAIVE_PAD, SEER_ROUTE_VARLEN_ONLY = 0, 1, 2
SEER_PATH_STATIC, SEER_PATH_VARLEN, SEER_PATH_EAGER = 0, 1, 2
SEER_REPACK_WINDOW_ONLY = 1
SEER_STATUS_V_RANGE = 1
SEER_ATTN_V_F16 = 1
SEER_MASK_NONE, SEER_MASK_CAUSAL, SEER_MASK_TREE = 0, 1, 2
SEER_PAGES_EXHAUSTED, SEER_PAGES_WIDTH, SEER_PAGES_INVALID = 1, 2, 4
SEER_ROPE_HALF, SEER_ROPE_PAIRS = 0, 1
SEER_ROPE_PLAIN, SEER_ROPE_LINEAR, SEER_ROPE_BASE, SEER_ROPE_BANDS, SEER_ROPE_RAMP = 0, 1, 2, 3, 4
SEER_ROPE_INVERSE = 1
SEER_EVICT_SHARED = 1
SEER_EVICT_ALIKE = 4

EXPORTED = ("seer_prepacked_bytes", "seer_prepack_weights", "seer_layer_workspace_bytes",
            "seer_layer_status_reset", "seer_layer_workspace_offsets", "seer_layer_forward_varlen",
            "seer_layer_forward_varlen_noalloc",
            "seer_layer_forward_varlen_timed", "seer_step0_detect", "seer_layer_forward_detect",
            "seer_layer_forward_detect_timed", "seer_batch_repack",
            "seer_layer_forward_cached", "seer_kv_export", "seer_graph_begin", "seer_graph_end",
            "seer_graph_launch", "seer_graph_destroy", "seer_lm_head_workspace_bytes", "seer_lm_head_prepack",
            "seer_lm_head_predict", "seer_remask_step", "seer_page_pool_bytes", "seer_page_plan", "seer_page_plan_latched",
            "seer_page_plan_kept", "seer_kv_store",
            "seer_attn_workspace_bytes", "seer_attn_prompt", "seer_attn_paged", "seer_rope_turns", "seer_rope_rows",
            "seer_kv_store_rope", "seer_row_positions", "seer_row_positions_kept", "seer_attn_weights_workspace_bytes", "seer_attn_weights",
            "seer_kv_evict_workspace_bytes", "seer_kv_evict", "seer_kv_evict_planned", "seer_last_error",
            "seer_abi_version")


class SeerError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("seer error %d: %s" % (code, msg))
        self.code = code


class seer_dims(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ff", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float)]


class seer_layer_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2")]


class seer_snr_params(ctypes.Structure):
    _fields_ = [("tau_num", ctypes.c_int32), ("tau_den", ctypes.c_int32),
                ("gamma_num", ctypes.c_int32), ("gamma_den", ctypes.c_int32),
                ("lookahead", ctypes.c_int32)]


class seer_repack_desc(ctypes.Structure):
    _fields_ = [("policy", ctypes.c_int32), ("tau_pad_num", ctypes.c_int32),
                ("tau_pad_den", ctypes.c_int32), ("granule", ctypes.c_int32),
                ("row_bytes", ctypes.c_int32), ("dst_capacity_rows", ctypes.c_int32),
                ("max_batch_hint", ctypes.c_int32), ("flags", ctypes.c_int32)]


class seer_route_ctrl(ctypes.Structure):
    _fields_ = [("total_rows", ctypes.c_int32), ("capacity_rows", ctypes.c_int32),
                ("n_static", ctypes.c_int32), ("n_varlen", ctypes.c_int32),
                ("n_eager", ctypes.c_int32), ("n_groups", ctypes.c_int32),
                ("max_alloc", ctypes.c_int32), ("status", ctypes.c_int32),
                ("ready", ctypes.c_int32), ("reserved", ctypes.c_int32 * 7)]


class seer_page_desc(ctypes.Structure):
    _fields_ = [("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("table_width", ctypes.c_int32)]


class seer_attn_desc(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("flags", ctypes.c_int32), ("scale", ctypes.c_float)]


class seer_rope_desc(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("original_len", ctypes.c_int32), ("theta", ctypes.c_float), ("factor", ctypes.c_float),
                ("low", ctypes.c_float), ("high", ctypes.c_float), ("magnitude", ctypes.c_float)]


_lib = None
_raw_stream = _current_device = None      # set by load_library
_P = ctypes.c_void_p
_I = ctypes.c_int32


def load_library():
    """Load libseer.so; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    # torch first: its HIP runtime carries the same soname, so the library binds
    # to the runtime that owns torch's streams and allocations.
    import torch  # noqa: F401
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libseer.so is not built (%s); run `python -m paper_2607_14557_amd.build`"
                           % LIB_PATH)
    global _raw_stream, _current_device
    _current_device = torch.cuda.current_device
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
        (lambda device: torch.cuda.current_stream(device).cuda_stream)
    L = ctypes.CDLL(LIB_PATH)
    L.seer_prepacked_bytes.argtypes = [ctypes.POINTER(seer_dims)]
    L.seer_prepacked_bytes.restype = ctypes.c_size_t
    L.seer_prepack_weights.argtypes = [ctypes.POINTER(seer_dims), ctypes.POINTER(seer_layer_weights),
                                       _P, ctypes.c_size_t, _P]
    L.seer_prepack_weights.restype = ctypes.c_int
    L.seer_layer_workspace_bytes.argtypes = [ctypes.POINTER(seer_dims), _I]
    L.seer_layer_workspace_bytes.restype = ctypes.c_size_t
    L.seer_layer_status_reset.argtypes = [_P, ctypes.c_size_t, _P]
    L.seer_layer_status_reset.restype = ctypes.c_int
    L.seer_layer_workspace_offsets.argtypes = [ctypes.POINTER(seer_dims), _I,
                                               ctypes.POINTER(ctypes.c_size_t)]
    L.seer_layer_workspace_offsets.restype = ctypes.c_int
    L.seer_layer_forward_varlen.argtypes = [ctypes.POINTER(seer_dims), _P, _P, _P, _I, _P, _P, _I,
                                            ctypes.c_float, _P, _P, ctypes.c_size_t, _P]
    L.seer_layer_forward_varlen.restype = ctypes.c_int
    L.seer_layer_forward_varlen_noalloc.argtypes = [ctypes.POINTER(seer_dims), _P, _P, _P, _I, _P, _P, _I,
                                                    ctypes.c_float, _P, _P, _P]
    L.seer_layer_forward_varlen_noalloc.restype = ctypes.c_int
    L.seer_layer_forward_varlen_timed.argtypes = L.seer_layer_forward_varlen.argtypes + [
        ctypes.POINTER(_P)]
    L.seer_layer_forward_varlen_timed.restype = ctypes.c_int
    L.seer_step0_detect.argtypes = [_P, _P, _P, _P, _I, _I, ctypes.POINTER(seer_snr_params), _P, _P, _P]
    L.seer_step0_detect.restype = ctypes.c_int
    L.seer_layer_forward_detect.argtypes = [ctypes.POINTER(seer_dims), _P, _P, _P, _I, _P, _I, ctypes.c_float,
                                            _P, _P, _P, ctypes.POINTER(seer_snr_params), _P, _P, _P,
                                            ctypes.c_size_t, _P]
    L.seer_layer_forward_detect.restype = ctypes.c_int
    L.seer_layer_forward_detect_timed.argtypes = L.seer_layer_forward_detect.argtypes + [ctypes.POINTER(_P)]
    L.seer_layer_forward_detect_timed.restype = ctypes.c_int
    L.seer_batch_repack.argtypes = [ctypes.POINTER(seer_repack_desc), ctypes.POINTER(_P),
                                    ctypes.POINTER(_P), _I, _P, _P, _P, _P, _I, _P, _P, _P, _P, _P, _P]
    L.seer_batch_repack.restype = ctypes.c_int
    L.seer_layer_forward_cached.argtypes = [ctypes.POINTER(seer_dims), _P, _P, _P, _I, _P, _P, _I,
                                            _P, _P, _I, _P, ctypes.c_size_t, _P]
    L.seer_layer_forward_cached.restype = ctypes.c_int
    L.seer_kv_export.argtypes = [ctypes.POINTER(seer_dims), _P, ctypes.c_size_t, _I, _P, _I, _P, _I, _P, _P]
    L.seer_kv_export.restype = ctypes.c_int
    L.seer_lm_head_workspace_bytes.argtypes = [ctypes.POINTER(seer_dims), _I, _I]
    L.seer_lm_head_workspace_bytes.restype = ctypes.c_size_t
    L.seer_lm_head_prepack.argtypes = [ctypes.POINTER(seer_dims), _P, _I, _P, ctypes.c_size_t, _P]
    L.seer_lm_head_prepack.restype = ctypes.c_int
    L.seer_lm_head_predict.argtypes = [ctypes.POINTER(seer_dims), _P, _I, _P, _I, _P, _I, _P, _P, _P,
                                       ctypes.c_size_t, _P]
    L.seer_lm_head_predict.restype = ctypes.c_int
    L.seer_remask_step.argtypes = [ctypes.POINTER(seer_dims), _P, _P, _I, _I, _I, _P, _P, _P, _P, _P, _I, _P, _P]
    L.seer_remask_step.restype = ctypes.c_int
    L.seer_graph_begin.argtypes = [_P]
    L.seer_graph_begin.restype = ctypes.c_int
    L.seer_graph_end.argtypes = [_P, ctypes.POINTER(_P)]
    L.seer_graph_end.restype = ctypes.c_int
    L.seer_graph_launch.argtypes = [_P, _P]
    L.seer_graph_launch.restype = ctypes.c_int
    L.seer_graph_destroy.argtypes = [_P]
    L.seer_graph_destroy.restype = ctypes.c_int
    heads, pages, _L = ctypes.POINTER(seer_attn_desc), ctypes.POINTER(seer_page_desc), ctypes.c_int64
    L.seer_page_pool_bytes.argtypes = [heads, pages]
    L.seer_page_pool_bytes.restype = ctypes.c_size_t
    L.seer_page_plan.argtypes = [pages, _P, _P, _P, _P, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P]
    L.seer_page_plan.restype = ctypes.c_int
    L.seer_page_plan_latched.argtypes = [pages, _P, _P, _P, _P, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P]
    L.seer_page_plan_latched.restype = ctypes.c_int
    L.seer_page_plan_kept.argtypes = [pages, _P, _P, _P, _P, _P, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P]
    L.seer_page_plan_kept.restype = ctypes.c_int
    L.seer_kv_store.argtypes = [heads, pages, _P, _L, _P, _L, _I, _P, _P, _P]
    L.seer_kv_store.restype = ctypes.c_int
    L.seer_attn_workspace_bytes.argtypes = [heads, _I, _I]
    L.seer_attn_workspace_bytes.restype = ctypes.c_size_t
    L.seer_attn_prompt.argtypes = [heads, _I, _P, _L, _P, _L, _P, _L, _P, _L, _I, _P, _P, _I, _P, ctypes.c_size_t, _P]
    L.seer_attn_prompt.restype = ctypes.c_int
    L.seer_attn_paged.argtypes = [heads, pages, _I, _P, _L, _P, _L, _I, _P, _P, _I, _P, _P, _P, _P, _I, _P,
                                  ctypes.c_size_t, _P]
    L.seer_attn_paged.restype = ctypes.c_int
    rope = ctypes.POINTER(seer_rope_desc)
    L.seer_rope_turns.argtypes = [rope, _I, ctypes.POINTER(ctypes.c_double)]
    L.seer_rope_turns.restype = ctypes.c_int
    L.seer_rope_rows.argtypes = [heads, rope, _P, _I, _P, _L, _P, _L, _P, _L, _P, _L, _I, _P, _P]
    L.seer_rope_rows.restype = ctypes.c_int
    L.seer_kv_store_rope.argtypes = [heads, pages, rope, _P, _P, _L, _P, _L, _P, _L, _P, _L, _I, _P, _P, _P, _P, _P, _P]
    L.seer_kv_store_rope.restype = ctypes.c_int
    L.seer_row_positions.argtypes = [_P, _P, _I, _P, _P, _P, _I, _P, _P, _P]
    L.seer_row_positions.restype = ctypes.c_int
    L.seer_row_positions_kept.argtypes = [_P, _P, _I, _P, _P, _P, _I, _P, _P, _P, _P, _P]
    L.seer_row_positions_kept.restype = ctypes.c_int
    L.seer_attn_weights_workspace_bytes.argtypes = [heads, pages, _I, _I]
    L.seer_attn_weights_workspace_bytes.restype = ctypes.c_size_t
    L.seer_attn_weights.argtypes = [heads, pages, _I, _P, _L, _I, _P, _P, _I, _I, _P, _P, _P, _P, _I, ctypes.c_float, _P,
                                    _P, _P, ctypes.c_size_t, _P]
    L.seer_attn_weights.restype = ctypes.c_int
    L.seer_kv_evict_workspace_bytes.argtypes = [heads, pages, _I]
    L.seer_kv_evict_workspace_bytes.restype = ctypes.c_size_t
    L.seer_kv_evict.argtypes = [heads, pages, _I, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t,
                                _P]
    L.seer_kv_evict.restype = ctypes.c_int
    L.seer_kv_evict_planned.argtypes = [heads, pages, _I, _P, _P, _P, _I, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P, _P,
                                        ctypes.c_size_t, _P]
    L.seer_kv_evict_planned.restype = ctypes.c_int
    L.seer_last_error.argtypes = []
    L.seer_last_error.restype = ctypes.c_char_p
    L.seer_abi_version.argtypes = []
    L.seer_abi_version.restype = ctypes.c_int32
    _lib = L
    return L


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(s):
    if s is None:
        # the current stream's handle, without the Stream object around it (0.2 us a call instead of 2.7)
        return _raw_stream(_current_device())
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _check(rc):
    if rc != 0:
        raise SeerError(rc, load_library().seer_last_error().decode())


def seer_last_error():
    return load_library().seer_last_error().decode()


def seer_abi_version():
    return load_library().seer_abi_version()


def seer_prepacked_bytes(dims):
    return load_library().seer_prepacked_bytes(ctypes.byref(dims))


def seer_prepack_weights(dims, weights, dst, dst_bytes=None, stream=None):
    """weights: dict with wq wk wv wo wg wu wd (device tensors) and optional g1 g2."""
    w = seer_layer_weights(*[_ptr(weights.get(n)) for n in
                             ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2")])
    nbytes = dst_bytes if dst_bytes is not None else dst.numel() * dst.element_size()
    _check(load_library().seer_prepack_weights(ctypes.byref(dims), ctypes.byref(w), _ptr(dst),
                                               nbytes, _stream(stream)))


def seer_layer_workspace_bytes(dims, max_rows):
    return load_library().seer_layer_workspace_bytes(ctypes.byref(dims), int(max_rows))


def seer_layer_status_reset(workspace, workspace_bytes=None, stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(load_library().seer_layer_status_reset(_ptr(workspace), nbytes, _stream(stream)))


def seer_layer_workspace_offsets(dims, max_rows):
    """Returns the eight byte offsets as a list."""
    off = (ctypes.c_size_t * 8)()
    _check(load_library().seer_layer_workspace_offsets(ctypes.byref(dims), int(max_rows), off))
    return list(off)


def seer_layer_forward_varlen_noalloc(dims, w_packed, x_in, x_out, total_rows_ub, cu_seqlens, seqused,
                                      batch, act_eps, act_count, status=None, stream=None):
    _check(load_library().seer_layer_forward_varlen_noalloc(
        ctypes.byref(dims), _ptr(w_packed), _ptr(x_in), _ptr(x_out), int(total_rows_ub), _ptr(cu_seqlens),
        _ptr(seqused), int(batch), float(act_eps), _ptr(act_count), _ptr(status), _stream(stream)))


def seer_layer_forward_varlen(dims, w_packed, x_in, x_out, total_rows_ub, cu_seqlens, seqused,
                              batch, act_eps, act_count, workspace, workspace_bytes=None,
                              stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(load_library().seer_layer_forward_varlen(
        ctypes.byref(dims), _ptr(w_packed), _ptr(x_in), _ptr(x_out), int(total_rows_ub),
        _ptr(cu_seqlens), _ptr(seqused), int(batch), float(act_eps), _ptr(act_count),
        _ptr(workspace), nbytes, _stream(stream)))


def seer_layer_forward_varlen_timed(dims, w_packed, x_in, x_out, total_rows_ub, cu_seqlens,
                                    seqused, batch, act_eps, act_count, workspace, events,
                                    workspace_bytes=None, stream=None):
    """events: sequence of 8 raw hipEvent_t handles (ints); a None entry
    skips that point."""
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    ev = (_P * 8)(*events)
    _check(load_library().seer_layer_forward_varlen_timed(
        ctypes.byref(dims), _ptr(w_packed), _ptr(x_in), _ptr(x_out), int(total_rows_ub),
        _ptr(cu_seqlens), _ptr(seqused), int(batch), float(act_eps), _ptr(act_count),
        _ptr(workspace), nbytes, _stream(stream), ev))


def seer_layer_forward_cached(dims, w_packed, x_in, x_out, total_rows_ub, cu_seqlens, seqused, batch,
                              kv_cache, cu_kv, kv_rows_ub, workspace, workspace_bytes=None, stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(load_library().seer_layer_forward_cached(
        ctypes.byref(dims), _ptr(w_packed), _ptr(x_in), _ptr(x_out), int(total_rows_ub),
        _ptr(cu_seqlens), _ptr(seqused), int(batch), _ptr(kv_cache), _ptr(cu_kv), int(kv_rows_ub),
        _ptr(workspace), nbytes, _stream(stream)))


def seer_kv_export(dims, workspace, total_rows_ub, cu_seqlens, batch, cu_kv, kv_rows_ub, kv_dst,
                   workspace_bytes=None, stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(load_library().seer_kv_export(
        ctypes.byref(dims), _ptr(workspace), nbytes, int(total_rows_ub), _ptr(cu_seqlens), int(batch),
        _ptr(cu_kv), int(kv_rows_ub), _ptr(kv_dst), _stream(stream)))


def seer_step0_detect(act_count, cu_seqlens, win_off, win_len, batch, d_ff, params, boundary,
                      keep_len, stream=None):
    _check(load_library().seer_step0_detect(
        _ptr(act_count), _ptr(cu_seqlens), _ptr(win_off), _ptr(win_len), int(batch), int(d_ff),
        ctypes.byref(params), _ptr(boundary), _ptr(keep_len), _stream(stream)))


def seer_layer_forward_detect(dims, w_packed, x_in, x_out, total_rows_ub, cu_seqlens, batch, act_eps,
                              act_count, win_off, win_len, params, boundary, keep_len, workspace,
                              workspace_bytes=None, stream=None, events=None):
    """The detection layer; with events (9 raw hipEvent_t handles) the timed
    variant."""
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    args = [ctypes.byref(dims), _ptr(w_packed), _ptr(x_in), _ptr(x_out), int(total_rows_ub), _ptr(cu_seqlens),
            int(batch), float(act_eps), _ptr(act_count), _ptr(win_off), _ptr(win_len), ctypes.byref(params),
            _ptr(boundary), _ptr(keep_len), _ptr(workspace), nbytes, _stream(stream)]
    L = load_library()
    if events is None:
        _check(L.seer_layer_forward_detect(*args))
    else:
        _check(L.seer_layer_forward_detect_timed(*args, (_P * 9)(*events)))


def seer_batch_repack(desc, srcs, dsts, cu_src, win_off, win_len, keep_len, batch, cu_dst,
                      seqused, route, ctrl_dev=None, ctrl_host=None, stream=None):
    n = len(srcs)
    src_arr = (_P * n)(*[_ptr(s) for s in srcs])
    dst_arr = (_P * n)(*[_ptr(d) for d in dsts])
    _check(load_library().seer_batch_repack(
        ctypes.byref(desc), src_arr, dst_arr, n, _ptr(cu_src), _ptr(win_off), _ptr(win_len),
        _ptr(keep_len), int(batch), _ptr(cu_dst), _ptr(seqused), _ptr(route), _ptr(ctrl_dev),
        _ptr(ctrl_host), _stream(stream)))


def seer_graph_begin(stream):
    """Start recording the seer calls issued on `stream` (a created stream)."""
    _check(load_library().seer_graph_begin(_stream(stream)))


def seer_graph_end(stream):
    """End the recording; returns the graph handle (an int)."""
    g = _P()
    _check(load_library().seer_graph_end(_stream(stream), ctypes.byref(g)))
    return g.value


def seer_graph_launch(graph, stream=None):
    _check(load_library().seer_graph_launch(graph, _stream(stream)))


def seer_graph_destroy(graph):
    _check(load_library().seer_graph_destroy(graph))


def seer_lm_head_workspace_bytes(dims, vocab, rows_ub):
    return load_library().seer_lm_head_workspace_bytes(ctypes.byref(dims), int(vocab), int(rows_ub))


def seer_lm_head_prepack(dims, w_lm, vocab, dst, dst_bytes=None, stream=None):
    nbytes = dst_bytes if dst_bytes is not None else dst.numel() * dst.element_size()
    _check(load_library().seer_lm_head_prepack(ctypes.byref(dims), _ptr(w_lm), int(vocab), _ptr(dst), nbytes,
                                               _stream(stream)))


def seer_lm_head_predict(dims, w_packed, vocab, x, rows_ub, cu_seqlens, batch, pred, conf, workspace,
                         workspace_bytes=None, stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(load_library().seer_lm_head_predict(
        ctypes.byref(dims), _ptr(w_packed), int(vocab), _ptr(x), int(rows_ub), _ptr(cu_seqlens), int(batch),
        _ptr(pred), _ptr(conf), _ptr(workspace), nbytes, _stream(stream)))


def seer_remask_step(dims, cu_seqlens, seqused, batch, max_used, steps_left, pred, conf, tokens, x0, emb, vocab,
                     x_next, stream=None):
    _check(load_library().seer_remask_step(
        ctypes.byref(dims), _ptr(cu_seqlens), _ptr(seqused), int(batch), int(max_used), int(steps_left),
        _ptr(pred), _ptr(conf), _ptr(tokens), _ptr(x0), _ptr(emb), int(vocab), _ptr(x_next), _stream(stream)))


def seer_page_pool_bytes(desc, pages):
    return load_library().seer_page_pool_bytes(ctypes.byref(desc), ctypes.byref(pages))


def seer_page_plan(pages, held, keep, cu_seqlens, seqused, batch, rows_ub, free_pages, free_in, free_out, table,
                   kv_len, slots, status, stream=None):
    _check(load_library().seer_page_plan(
        ctypes.byref(pages), _ptr(held), _ptr(keep), _ptr(cu_seqlens), _ptr(seqused), int(batch), int(rows_ub),
        _ptr(free_pages), _ptr(free_in), _ptr(free_out), _ptr(table), _ptr(kv_len), _ptr(slots), _ptr(status),
        _stream(stream)))


def seer_page_plan_latched(pages, held, keep, cu_seqlens, seqused, batch, rows_ub, free_pages, free_in, free_out, table,
                           kv_len, slots, status, refused, stream=None, kept=None):
    """With kept: seer_page_plan_kept."""
    args = (_ptr(keep), _ptr(cu_seqlens), _ptr(seqused), int(batch), int(rows_ub), _ptr(free_pages), _ptr(free_in),
            _ptr(free_out), _ptr(table), _ptr(kv_len), _ptr(slots), _ptr(status), _ptr(refused), _stream(stream))
    if kept is None:
        _check(load_library().seer_page_plan_latched(ctypes.byref(pages), _ptr(held), *args))
    else:
        _check(load_library().seer_page_plan_kept(ctypes.byref(pages), _ptr(held), _ptr(kept), *args))


def seer_kv_store(desc, pages, k, k_stride, v, v_stride, rows_ub, slots, pool, stream=None):
    """k_stride, v_stride: elements from one row to the next."""
    _check(load_library().seer_kv_store(
        ctypes.byref(desc), ctypes.byref(pages), _ptr(k), int(k_stride), _ptr(v), int(v_stride), int(rows_ub),
        _ptr(slots), _ptr(pool), _stream(stream)))


def seer_attn_workspace_bytes(desc, rows_ub, batch):
    return load_library().seer_attn_workspace_bytes(ctypes.byref(desc), int(rows_ub), int(batch))


def seer_attn_prompt(desc, mask, q, q_stride, k, k_stride, v, v_stride, out, out_stride, rows_ub, cu_seqlens,
                     seqused, batch, workspace, workspace_bytes=None, stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(load_library().seer_attn_prompt(
        ctypes.byref(desc), int(mask), _ptr(q), int(q_stride), _ptr(k), int(k_stride), _ptr(v), int(v_stride),
        _ptr(out), int(out_stride), int(rows_ub), _ptr(cu_seqlens), _ptr(seqused), int(batch), _ptr(workspace),
        nbytes, _stream(stream)))


def seer_attn_paged(desc, pages, mask, q, q_stride, out, out_stride, rows_ub, cu_seqlens, seqused, batch, pool, table,
                    kv_len, tree_bits, tree_words, workspace, workspace_bytes=None, stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(load_library().seer_attn_paged(
        ctypes.byref(desc), ctypes.byref(pages), int(mask), _ptr(q), int(q_stride), _ptr(out), int(out_stride),
        int(rows_ub), _ptr(cu_seqlens), _ptr(seqused), int(batch), _ptr(pool), _ptr(table), _ptr(kv_len),
        _ptr(tree_bits), int(tree_words), _ptr(workspace), nbytes, _stream(stream)))


def seer_rope_turns(rope, head_dim):
    """The frequencies as a list of turns a position; runs on the host."""
    out = (ctypes.c_double * 64)()
    _check(load_library().seer_rope_turns(ctypes.byref(rope), int(head_dim), out))
    return list(out)[:(rope.rotary_dim or int(head_dim)) // 2]


def _rope(rope):
    return None if rope is None else ctypes.byref(rope)


def seer_rope_rows(desc, rope, turns, flags, q, q_stride, k, k_stride, q_out, q_out_stride, k_out, k_out_stride, rows_ub,
                   positions, stream=None):
    """turns: fp64 device tensor of seer_rope_turns."""
    _check(load_library().seer_rope_rows(
        ctypes.byref(desc), _rope(rope), _ptr(turns), int(flags), _ptr(q), int(q_stride), _ptr(k), int(k_stride),
        _ptr(q_out), int(q_out_stride), _ptr(k_out), int(k_out_stride), int(rows_ub), _ptr(positions), _stream(stream)))


def seer_kv_store_rope(desc, pages, rope, turns, q, q_stride, q_out, q_out_stride, k, k_stride, v, v_stride, rows_ub,
                       positions, slots, pool, weight, number, stream=None):
    _check(load_library().seer_kv_store_rope(
        ctypes.byref(desc), ctypes.byref(pages), _rope(rope), _ptr(turns), _ptr(q), int(q_stride), _ptr(q_out),
        int(q_out_stride), _ptr(k), int(k_stride), _ptr(v), int(v_stride), int(rows_ub), _ptr(positions), _ptr(slots),
        _ptr(pool), _ptr(weight), _ptr(number), _stream(stream)))


def seer_row_positions(cu_seqlens, seqused, batch, seen, base, status, rows_ub, positions, next, stream=None, kv_len=None,
                       kept=None):
    """With kept: seer_row_positions_kept."""
    args = (_ptr(cu_seqlens), _ptr(seqused), int(batch), _ptr(seen), _ptr(base), _ptr(status), int(rows_ub), _ptr(positions),
            _ptr(next))
    if kept is None:
        _check(load_library().seer_row_positions(*args, _stream(stream)))
    else:
        _check(load_library().seer_row_positions_kept(*args, _ptr(kv_len), _ptr(kept), _stream(stream)))


def seer_attn_weights_workspace_bytes(desc, pages, rows_ub, batch):
    return load_library().seer_attn_weights_workspace_bytes(ctypes.byref(desc), ctypes.byref(pages), int(rows_ub),
                                                            int(batch))


def seer_attn_weights(desc, pages, mask, q, q_stride, rows_ub, cu_seqlens, seqused, batch, last, pool, table, kv_len,
                      tree_bits, tree_words, decay, prev, weight, workspace, workspace_bytes=None, stream=None):
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    _check(load_library().seer_attn_weights(
        ctypes.byref(desc), ctypes.byref(pages), int(mask), _ptr(q), int(q_stride), int(rows_ub), _ptr(cu_seqlens),
        _ptr(seqused), int(batch), int(last), _ptr(pool), _ptr(table), _ptr(kv_len), _ptr(tree_bits), int(tree_words),
        float(decay), _ptr(prev), _ptr(weight), _ptr(workspace), nbytes, _stream(stream)))


def seer_kv_evict_workspace_bytes(desc, pages, batch):
    return load_library().seer_kv_evict_workspace_bytes(ctypes.byref(desc), ctypes.byref(pages), int(batch))


def seer_kv_evict(desc, pages, flags, kv_len, budget, seen, batch, first, recent, table, pool, weight, number, weight_out,
                  number_out, kept, workspace, workspace_bytes=None, stream=None, status=None):
    """With status: seer_kv_evict_planned."""
    nbytes = workspace_bytes if workspace_bytes is not None else workspace.numel() * workspace.element_size()
    args = (ctypes.byref(desc), ctypes.byref(pages), int(flags), _ptr(kv_len), _ptr(budget), _ptr(seen), int(batch), int(first),
            int(recent), _ptr(table), _ptr(pool), _ptr(weight), _ptr(number), _ptr(weight_out), _ptr(number_out), _ptr(kept))
    if status is None:
        _check(load_library().seer_kv_evict(*args, _ptr(workspace), nbytes, _stream(stream)))
    else:
        _check(load_library().seer_kv_evict_planned(*args, _ptr(status), _ptr(workspace), nbytes, _stream(stream)))
