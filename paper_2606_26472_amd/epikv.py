"""Python binding of libepikv.so (ctypes).

Argument marshalling only: every step of the eviction path, and of filling and
reading the cache, runs in the HIP kernels behind the C ABI declared in include/epikv.h.  torch tensors supply
device memory (``data_ptr``) and the current HIP stream.  The library must be
built (``python -m paper_2606_26472_amd.build``); there is no fallback.
"""
from __future__ import annotations

import array
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
# EPIKV_LIB selects another build of the same library (e.g. the host-ASan
# one); a missing file is an error like a missing default build.
LIB_PATH = os.environ.get("EPIKV_LIB") or os.path.join(_HERE, "libepikv.so")

# status codes (include/epikv.h)
EPIKV_OK = 0
EPIKV_EINVAL_NULL = -1
EPIKV_EINVAL_SHAPE = -2
EPIKV_EINVAL_PARAM = -3
EPIKV_EALIGN = -4
EPIKV_EWORKSPACE = -5
EPIKV_EALIAS = -6
EPIKV_ELAUNCH = -7

SEQ_OK = 0
SEQ_BUDGET = 1
SEQ_RANGE = 2
SEQ_SYNC = 3
COMPACT_OUT_OF_PLACE, COMPACT_IN_PLACE, COMPACT_REMAP = 0, 1, 2

SIGNAL_HS = 0
SIGNAL_LAGKV = 1
SIGNAL_KV_KEY = 2
SIGNAL_KV_VAL = 3
SIGNAL_LAGKV_KEY = 4
SMOOTH_Z = 0
SMOOTH_MEAN = 1
SMOOTH_RAW = 2
SMOOTH_EMA = 3
MAX_BAND = 32
KV_BF16, KV_MXFP4 = 0, 1
DTYPE_BF16, DTYPE_FP32 = 0, 1
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
AXES_SECTIONS, AXES_TURNS = 0, 1
AXES_SHARED, AXES_APART = 0, 1
MAX_AXES = 4
ROPE_PLAIN, ROPE_LINEAR, ROPE_NTK, ROPE_BANDS, ROPE_YARN = 0, 1, 2, 3, 4

EXPORTED = ("epikv_default_cfg", "epikv_strerror", "epikv_check_cfg",
            "epikv_state_bytes", "epikv_state_layout",
            "epikv_workspace_bytes", "epikv_compact_workspace_bytes",
            "epikv_state_init", "epikv_score", "epikv_score_tokens",
            "epikv_zscore", "epikv_select", "epikv_select_workspace_bytes",
            "epikv_select_ws", "epikv_compact",
            "epikv_compact_inplace", "epikv_compact_remap",
            "epikv_evict_step", "epikv_evict_step_noalloc",
            "epikv_kv_row_bytes", "epikv_default_rope", "epikv_check_rope",
            "epikv_rope_table_bytes", "epikv_rope_table", "epikv_rope",
            "epikv_append", "epikv_read", "epikv_attend_workspace_bytes",
            "epikv_attend", "epikv_cfg_bytes", "epikv_check_axes",
            "epikv_rope_axes_table", "epikv_rope_axes", "epikv_append_axes",
            "epikv_attend_weigh_workspace_bytes", "epikv_attend_weigh")


class EpikvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


class Cfg(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_band_a", ctypes.c_int32), ("n_band_b", ctypes.c_int32),
                ("window", ctypes.c_int32), ("eps", ctypes.c_float),
                ("signal", ctypes.c_int32), ("smoothing", ctypes.c_int32),
                ("budget", ctypes.c_int32), ("recent", ctypes.c_int32),
                ("ema_alpha", ctypes.c_float),
                ("kv_format", ctypes.c_int32)]


class Pool(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("stride_layer", ctypes.c_int64),
                ("stride_kv", ctypes.c_int64), ("stride_page", ctypes.c_int64),
                ("n_pages", ctypes.c_int64)]


class StepIO(ctypes.Structure):
    _fields_ = [("chunk", ctypes.c_int32),
                ("hidden", ctypes.POINTER(ctypes.c_void_p)),
                ("ld_tok", ctypes.c_int64), ("ld_seq", ctypes.c_int64),
                ("n_cached", ctypes.c_void_p), ("n_prefix", ctypes.c_void_p),
                ("src", Pool), ("src_pt", ctypes.c_void_p),
                ("ld_src_pt", ctypes.c_int64),
                ("dst", Pool), ("dst_pt", ctypes.c_void_p),
                ("ld_dst_pt", ctypes.c_int64),
                ("scores", ctypes.c_void_p), ("dst_scores", ctypes.c_void_p),
                ("src_pos", ctypes.c_void_p), ("dst_pos", ctypes.c_void_p),
                ("ld_s", ctypes.c_int64),
                ("state_in", ctypes.c_void_p), ("state_out", ctypes.c_void_p),
                ("keep_idx", ctypes.c_void_p), ("n_keep", ctypes.c_void_p),
                ("seq_status", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t),
                ("in_place", ctypes.c_int32)]


class Rows(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("ld_seq", ctypes.c_int64),
                ("ld_tok", ctypes.c_int64), ("ld_head", ctypes.c_int64)]


class Rope(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("scaling", ctypes.c_int32), ("n_pos", ctypes.c_int32),
                ("original", ctypes.c_int32), ("theta", ctypes.c_float),
                ("factor", ctypes.c_float), ("turns_low", ctypes.c_float),
                ("turns_high", ctypes.c_float), ("amplitude", ctypes.c_float)]


class Axes(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32),
                ("pairs", ctypes.c_int32 * MAX_AXES),
                ("order", ctypes.c_int32), ("frequencies", ctypes.c_int32)]


class AppendIO(ctypes.Structure):
    _fields_ = [("chunk", ctypes.c_int32), ("layer", ctypes.c_int32),
                ("pool", Pool), ("page_table", ctypes.c_void_p),
                ("ld_pt", ctypes.c_int64), ("n_cached", ctypes.c_void_p),
                ("n_new", ctypes.c_void_p), ("k", Rows), ("v", Rows),
                ("rope", ctypes.POINTER(Rope)),
                ("rope_table", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("ld_pos", ctypes.c_int64),
                ("n_heads", ctypes.c_int32), ("q", Rows), ("q_out", Rows),
                ("pos", ctypes.c_void_p), ("ld_s", ctypes.c_int64),
                ("seq_status", ctypes.c_void_p)]


class ReadIO(ctypes.Structure):
    _fields_ = [("chunk", ctypes.c_int32), ("layer", ctypes.c_int32),
                ("pool", Pool), ("page_table", ctypes.c_void_p),
                ("ld_pt", ctypes.c_int64), ("first", ctypes.c_void_p),
                ("k", Rows), ("v", Rows), ("seq_status", ctypes.c_void_p)]


class AttendIO(ctypes.Structure):
    _fields_ = [("chunk", ctypes.c_int32), ("layer", ctypes.c_int32),
                ("pool", Pool), ("page_table", ctypes.c_void_p),
                ("ld_pt", ctypes.c_int64), ("n_cached", ctypes.c_void_p),
                ("n_new", ctypes.c_void_p), ("n_heads", ctypes.c_int32),
                ("q", Rows), ("out", Rows), ("lse", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("seq_status", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class WeighIO(ctypes.Structure):
    _fields_ = [("old", ctypes.c_void_p), ("weights", ctypes.c_void_p),
                ("ld_s", ctypes.c_int64), ("keep_old", ctypes.c_float),
                ("keep_new", ctypes.c_float), ("gain", ctypes.c_float),
                ("watch", ctypes.c_int32)]


_lib = None


def _same_cfg(nbytes):
    if nbytes != ctypes.sizeof(Cfg):
        raise RuntimeError(f"{LIB_PATH}: its epikv_cfg has {nbytes} bytes, this binding's {ctypes.sizeof(Cfg)}: "
                           "build the library anew")


def lib() -> ctypes.CDLL:
    """Load libepikv.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build the HIP library first "
            "(python -m paper_2606_26472_amd.build)")
    # The device buffers handed to the library are torch's, and the torch
    # wheel carries its own HIP runtime under the same soname as the
    # system's (libamdhip64.so.7).  Importing torch first makes the library
    # bind to that runtime; opened first, it would bring in the system copy
    # as a second runtime, whose launches fail on torch's allocations.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    L = ctypes.CDLL(LIB_PATH)
    P = ctypes.c_void_p
    i32, i64, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    cfgp = ctypes.POINTER(Cfg)
    poolp = ctypes.POINTER(Pool)
    ropep, rowsp = ctypes.POINTER(Rope), ctypes.POINTER(Rows)
    axesp = ctypes.POINTER(Axes)
    sig = {
        "epikv_default_cfg": (ctypes.c_int, [cfgp]),
        "epikv_strerror": (ctypes.c_char_p, [ctypes.c_int]),
        "epikv_check_cfg": (ctypes.c_int, [cfgp]),
        "epikv_state_bytes": (sz, [cfgp]),
        "epikv_state_layout": (ctypes.c_int, [cfgp, ctypes.POINTER(sz)]),
        "epikv_workspace_bytes": (sz, [cfgp, i32]),
        "epikv_compact_workspace_bytes": (sz, [cfgp]),
        "epikv_state_init": (ctypes.c_int, [cfgp, P, P]),
        "epikv_score": (ctypes.c_int, [cfgp, i32, P, i64, i64,
                                       poolp, P, i64, P, P, P, P, P, sz, P]),
        "epikv_zscore": (ctypes.c_int, [cfgp, i32, P, P, P, P, P, i64, P, P]),
        "epikv_score_tokens": (ctypes.c_int, [cfgp, i32, P, i64,
                                              i64, P, P, P, P, i64, P]),
        "epikv_select": (ctypes.c_int, [cfgp, P, i64, P, P, P, P, P, P]),
        "epikv_select_workspace_bytes": (sz, [cfgp]),
        "epikv_select_ws": (ctypes.c_int, [cfgp, P, i64, P, P, P, P, P, P,
                                           sz, P]),
        "epikv_compact": (ctypes.c_int, [cfgp, poolp, P, i64, poolp, P, i64,
                                         P, P, P, P, P, P, i64, P, P, sz, P]),
        "epikv_compact_inplace": (ctypes.c_int, [cfgp, poolp, P, i64, P, P,
                                                 P, P, i64, P, P, sz, P]),
        "epikv_compact_remap": (ctypes.c_int, [cfgp, poolp, P, i64, P, P,
                                               P, P, i64, P, P, sz, P]),
        "epikv_evict_step": (ctypes.c_int, [cfgp, ctypes.POINTER(StepIO), P]),
        "epikv_evict_step_noalloc": (ctypes.c_int,
                                     [cfgp, ctypes.POINTER(StepIO), P]),
        "epikv_cfg_bytes": (sz, []),
        "epikv_kv_row_bytes": (sz, [cfgp]),
        "epikv_default_rope": (ctypes.c_int, [ropep]),
        "epikv_check_rope": (ctypes.c_int, [ropep]),
        "epikv_rope_table_bytes": (sz, [ropep]),
        "epikv_rope_table": (ctypes.c_int, [ropep, P, P]),
        "epikv_rope": (ctypes.c_int, [ropep, P, i32, i32, i32, i32, i32, rowsp,
                                      rowsp, P, i64, i32, P, P]),
        "epikv_append": (ctypes.c_int, [cfgp, ctypes.POINTER(AppendIO), P]),
        "epikv_read": (ctypes.c_int, [cfgp, ctypes.POINTER(ReadIO), P]),
        "epikv_attend_workspace_bytes": (sz, [cfgp, i32, i32]),
        "epikv_attend": (ctypes.c_int, [cfgp, ctypes.POINTER(AttendIO), P]),
        "epikv_check_axes": (ctypes.c_int, [ropep, axesp]),
        "epikv_rope_axes_table": (ctypes.c_int, [ropep, axesp, P, P]),
        "epikv_rope_axes": (ctypes.c_int, [ropep, axesp, P, i32, i32, i32, i32,
                                           i32, rowsp, rowsp, P, i64, i32, P,
                                           P]),
        "epikv_append_axes": (ctypes.c_int, [cfgp, ctypes.POINTER(AppendIO),
                                             axesp, P, i64, P]),
        "epikv_attend_weigh_workspace_bytes": (sz, [cfgp, i32, i32, i64, i32]),
        "epikv_attend_weigh": (ctypes.c_int, [cfgp, ctypes.POINTER(AttendIO),
                                              ctypes.POINTER(WeighIO), P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _same_cfg(L.epikv_cfg_bytes())
    _lib = L
    return L


def strerror(status: int) -> str:
    return lib().epikv_strerror(int(status)).decode()


def _check(status: int, where: str):
    if status != EPIKV_OK:
        raise EpikvError(status, where)


def _ptr(t):
    """Device (or host) address of a tensor, or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _ws(t, nbytes):
    """Address of a workspace tensor, refusing one smaller than the size
    that will be declared to the library (it would write past its end)."""
    if t is not None and not isinstance(t, int):
        have = t.numel() * t.element_size()
        if have < int(nbytes):
            raise ValueError(f"workspace tensor holds {have} bytes, "
                             f"{int(nbytes)} declared")
    return _ptr(t)


def _stream(stream):
    if stream is None:
        import torch
        if torch.cuda.is_initialized():
            # (the handle alone: building a Stream object costs 1 us; the
            # names are private, and a torch without them takes that way)
            try:
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
            except AttributeError:
                pass
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ---------------------------------------------------------------------------
# Configuration and sizes
# ---------------------------------------------------------------------------
def default_cfg(**overrides) -> Cfg:
    c = Cfg()
    _check(lib().epikv_default_cfg(ctypes.byref(c)), "epikv_default_cfg")
    for k, v in overrides.items():
        setattr(c, k, v)
    return c


def check_cfg(cfg: Cfg) -> int:
    return lib().epikv_check_cfg(ctypes.byref(cfg))


def state_bytes(cfg: Cfg) -> int:
    return int(lib().epikv_state_bytes(ctypes.byref(cfg)))


def state_layout(cfg: Cfg):
    off = (ctypes.c_size_t * 5)()
    _check(lib().epikv_state_layout(ctypes.byref(cfg), off),
           "epikv_state_layout")
    return [int(x) for x in off]


def workspace_bytes(cfg: Cfg, chunk: int) -> int:
    return int(lib().epikv_workspace_bytes(ctypes.byref(cfg), int(chunk)))


def compact_workspace_bytes(cfg: Cfg) -> int:
    return int(lib().epikv_compact_workspace_bytes(ctypes.byref(cfg)))


def select_workspace_bytes(cfg: Cfg) -> int:
    return int(lib().epikv_select_workspace_bytes(ctypes.byref(cfg)))


def kv_row_bytes(cfg: Cfg) -> int:
    return int(lib().epikv_kv_row_bytes(ctypes.byref(cfg)))


def attend_workspace_bytes(cfg: Cfg, chunk: int, n_heads: int) -> int:
    return int(lib().epikv_attend_workspace_bytes(ctypes.byref(cfg), int(chunk),
                                                  int(n_heads)))


def attend_weigh_workspace_bytes(cfg: Cfg, chunk: int, n_heads: int,
                                 ld_pt: int, watch: int = 0) -> int:
    return int(lib().epikv_attend_weigh_workspace_bytes(
        ctypes.byref(cfg), int(chunk), int(n_heads), int(ld_pt), int(watch)))


def axes_of(pairs, order=AXES_SECTIONS, frequencies=AXES_SHARED) -> Axes:
    """epikv_axes with so many pairs of each axis."""
    pairs = [int(n) for n in pairs]
    if len(pairs) > MAX_AXES:
        raise ValueError(f"{len(pairs)} axes, {MAX_AXES} at most")
    return Axes(len(pairs), (ctypes.c_int32 * MAX_AXES)(*pairs), int(order), int(frequencies))


def check_axes(rope: Rope, axes: Axes) -> int:
    return lib().epikv_check_axes(ctypes.byref(rope), ctypes.byref(axes))


def default_rope(**overrides) -> Rope:
    r = Rope()
    _check(lib().epikv_default_rope(ctypes.byref(r)), "epikv_default_rope")
    for k, v in overrides.items():
        setattr(r, k, v)
    return r


def check_rope(rope: Rope) -> int:
    return lib().epikv_check_rope(ctypes.byref(rope))


def rope_table_bytes(rope: Rope) -> int:
    return int(lib().epikv_rope_table_bytes(ctypes.byref(rope)))


def rows_of(t) -> Rows:
    """epikv_rows describing a [B][chunk][heads][head_dim] tensor (any
    strides, channels adjacent); None gives a NULL base."""
    if t is None:
        return Rows(None, 0, 0, 0)
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError("rows need a [batch][chunk][heads][head_dim] tensor "
                         "with adjacent channels")
    # (the stride of an axis of one entry means nothing)
    s = [t.stride(i) if t.shape[i] > 1 else 0 for i in range(3)]
    return Rows(t.data_ptr(), s[0], s[1], s[2])


def pool_of(t) -> Pool:
    """epikv_pool describing a tensor laid out [L][2][n_pages][page][H][d]
    (4-bit rows: uint8 [L][2][n_pages][page][row_bytes])."""
    es = t.element_size()
    L, two, n_pages = t.shape[0], t.shape[1], t.shape[2]
    assert two == 2
    s = t.stride()
    return Pool(t.data_ptr(), s[0] * es, s[1] * es, s[2] * es, n_pages)


# ---------------------------------------------------------------------------
# Entry points (same names as the C ABI)
# ---------------------------------------------------------------------------
def epikv_state_init(cfg: Cfg, state, stream=None):
    _check(lib().epikv_state_init(ctypes.byref(cfg), _ptr(state),
                                  _stream(stream)), "epikv_state_init")


def _hidden_array(hidden):
    """The layers' addresses as a host array (kept alive by the caller)."""
    if hidden is None:
        return None
    # (a packed array: building a ctypes one of 15 addresses took as long as
    # the rest of the binding's call)
    try:
        return array.array("Q", [h.data_ptr() for h in hidden])
    except AttributeError:
        return array.array("Q", [_ptr(h) or 0 for h in hidden])


def _address(arr):
    return None if arr is None else arr.buffer_info()[0]


def _every_layer(cfg: Cfg, arr, where):
    """The library reads one address per band layer from the host array."""
    if arr is None or cfg.signal != SIGNAL_HS:
        return
    want = cfg.n_band_a + cfg.n_band_b
    if len(arr) < want:
        raise ValueError(f"{where}: hidden states of {len(arr)} layers, cfg has {want} band layers")


def epikv_score(cfg: Cfg, chunk: int, hidden=None, ld_tok=0, ld_seq=0,
                pool: Pool | None = None, page_table=None, ld_pt=0,
                n_cached=None, state_in=None, state_out=None, sig=None,
                workspace=None, workspace_bytes_=0, stream=None):
    arr = _hidden_array(hidden)
    _every_layer(cfg, arr, "epikv_score")
    _check(lib().epikv_score(
        ctypes.byref(cfg), int(chunk), _address(arr), int(ld_tok), int(ld_seq),
        ctypes.byref(pool) if pool is not None else None, _ptr(page_table),
        int(ld_pt), _ptr(n_cached), _ptr(state_in), _ptr(state_out),
        _ptr(sig), _ws(workspace, workspace_bytes_), int(workspace_bytes_),
        _stream(stream)),
        "epikv_score")


def epikv_zscore(cfg: Cfg, chunk: int, sig, n_cached, state_in, state_out,
                 scores, ld_s, smoothed=None, stream=None):
    _check(lib().epikv_zscore(
        ctypes.byref(cfg), int(chunk), _ptr(sig), _ptr(n_cached),
        _ptr(state_in), _ptr(state_out), _ptr(scores), int(ld_s),
        _ptr(smoothed), _stream(stream)), "epikv_zscore")


def epikv_score_tokens(cfg: Cfg, chunk: int, hidden, ld_tok, ld_seq, n_cached,
                       state_in, state_out, scores, ld_s, stream=None):
    arr = _hidden_array(hidden)
    _every_layer(cfg, arr, "epikv_score_tokens")
    _check(lib().epikv_score_tokens(
        ctypes.byref(cfg), int(chunk), _address(arr), int(ld_tok), int(ld_seq),
        _ptr(n_cached), _ptr(state_in), _ptr(state_out), _ptr(scores),
        int(ld_s), _stream(stream)), "epikv_score_tokens")


def epikv_select(cfg: Cfg, scores, ld_s, n_cached, n_prefix, keep_idx,
                 n_keep, seq_status, stream=None):
    _check(lib().epikv_select(
        ctypes.byref(cfg), _ptr(scores), int(ld_s), _ptr(n_cached),
        _ptr(n_prefix), _ptr(keep_idx), _ptr(n_keep), _ptr(seq_status),
        _stream(stream)), "epikv_select")


def epikv_select_ws(cfg: Cfg, scores, ld_s, n_cached, n_prefix, keep_idx,
                    n_keep, seq_status, workspace=None, workspace_bytes_=0,
                    stream=None):
    _check(lib().epikv_select_ws(
        ctypes.byref(cfg), _ptr(scores), int(ld_s), _ptr(n_cached),
        _ptr(n_prefix), _ptr(keep_idx), _ptr(n_keep), _ptr(seq_status),
        _ws(workspace, workspace_bytes_), int(workspace_bytes_),
        _stream(stream)),
        "epikv_select_ws")


def epikv_compact(cfg: Cfg, src: Pool, src_pt, ld_src_pt, dst: Pool, dst_pt,
                  ld_dst_pt, keep_idx, n_keep, src_scores=None,
                  dst_scores=None, src_pos=None, dst_pos=None, ld_s=0,
                  seq_status=None, workspace=None, workspace_bytes_=0,
                  stream=None):
    _check(lib().epikv_compact(
        ctypes.byref(cfg), ctypes.byref(src), _ptr(src_pt), int(ld_src_pt),
        ctypes.byref(dst), _ptr(dst_pt), int(ld_dst_pt), _ptr(keep_idx),
        _ptr(n_keep), _ptr(src_scores), _ptr(dst_scores), _ptr(src_pos),
        _ptr(dst_pos), int(ld_s), _ptr(seq_status),
        _ws(workspace, workspace_bytes_), int(workspace_bytes_),
        _stream(stream)),
        "epikv_compact")


def epikv_compact_inplace(cfg: Cfg, pool: Pool, page_table, ld_pt, keep_idx,
                          n_keep, scores=None, pos=None, ld_s=0,
                          seq_status=None, workspace=None, workspace_bytes_=0,
                          stream=None):
    _check(lib().epikv_compact_inplace(
        ctypes.byref(cfg), ctypes.byref(pool), _ptr(page_table), int(ld_pt),
        _ptr(keep_idx), _ptr(n_keep), _ptr(scores), _ptr(pos), int(ld_s),
        _ptr(seq_status), _ws(workspace, workspace_bytes_), int(workspace_bytes_),
        _stream(stream)), "epikv_compact_inplace")


def epikv_compact_remap(cfg: Cfg, pool: Pool, page_table, ld_pt, keep_idx,
                        n_keep, scores=None, pos=None, ld_s=0,
                        seq_status=None, workspace=None, workspace_bytes_=0,
                        stream=None):
    _check(lib().epikv_compact_remap(
        ctypes.byref(cfg), ctypes.byref(pool), _ptr(page_table), int(ld_pt),
        _ptr(keep_idx), _ptr(n_keep), _ptr(scores), _ptr(pos), int(ld_s),
        _ptr(seq_status), _ws(workspace, workspace_bytes_), int(workspace_bytes_),
        _stream(stream)), "epikv_compact_remap")


def make_step_io(chunk, hidden, ld_tok, ld_seq, n_cached, n_prefix,
                 src: Pool, src_pt, ld_src_pt, dst: Pool, dst_pt, ld_dst_pt,
                 scores, ld_s, state_in, state_out, keep_idx, n_keep,
                 seq_status, workspace, workspace_bytes_, dst_scores=None,
                 src_pos=None, dst_pos=None, in_place=False) -> StepIO:
    """Build the epikv_step_io struct.  The returned object holds references
    to every tensor (and the hidden pointer array) it was built from, so a
    temporary passed here cannot be freed while the struct is in use."""
    io = StepIO()
    io._tensors_keepalive = [n_cached, n_prefix, src_pt, dst_pt, scores,
                             state_in, state_out, keep_idx, n_keep,
                             seq_status, workspace, dst_scores, src_pos,
                             dst_pos, hidden]
    io.chunk = int(chunk)
    arr = _hidden_array(hidden)
    io._hidden_keepalive = arr
    io.hidden = ctypes.cast(_address(arr), ctypes.POINTER(ctypes.c_void_p)) \
        if arr is not None else None
    io.ld_tok, io.ld_seq = int(ld_tok), int(ld_seq)
    io.n_cached, io.n_prefix = _ptr(n_cached), _ptr(n_prefix)
    io.src, io.src_pt, io.ld_src_pt = src, _ptr(src_pt), int(ld_src_pt)
    io.dst, io.dst_pt, io.ld_dst_pt = dst, _ptr(dst_pt), int(ld_dst_pt)
    io.scores, io.dst_scores = _ptr(scores), _ptr(dst_scores)
    io.src_pos, io.dst_pos = _ptr(src_pos), _ptr(dst_pos)
    io.ld_s = int(ld_s)
    io.state_in, io.state_out = _ptr(state_in), _ptr(state_out)
    io.keep_idx, io.n_keep = _ptr(keep_idx), _ptr(n_keep)
    io.seq_status = _ptr(seq_status)
    io.workspace = _ws(workspace, workspace_bytes_)
    io.workspace_bytes = int(workspace_bytes_)
    io.in_place = int(in_place)   # False/True, or a COMPACT_* mode
    return io


def _step_layers(cfg: Cfg, io: StepIO, where):
    if io.chunk > 0:  # (a step without new tokens reads no hidden states)
        _every_layer(cfg, getattr(io, "_hidden_keepalive", None), where)


def epikv_evict_step(cfg: Cfg, io: StepIO, stream=None):
    _step_layers(cfg, io, "epikv_evict_step")
    _check(lib().epikv_evict_step(ctypes.byref(cfg), ctypes.byref(io),
                                  _stream(stream)), "epikv_evict_step")


def epikv_evict_step_noalloc(cfg: Cfg, io: StepIO, stream=None):
    """epikv_evict_step with the library's per-GPU scratch array
    (io.workspace is ignored)."""
    _step_layers(cfg, io, "epikv_evict_step_noalloc")
    _check(lib().epikv_evict_step_noalloc(ctypes.byref(cfg), ctypes.byref(io),
                                          _stream(stream)),
           "epikv_evict_step_noalloc")


# ---------------------------------------------------------------------------
# Filling and reading the cache
# ---------------------------------------------------------------------------
def _expect(t, dtype, shape, what):
    """A wrong type or shape would be read or written past its end."""
    if t is None or isinstance(t, Rows):
        return
    import torch
    want = getattr(torch, dtype)
    if t.dtype not in (want, torch.int16 if dtype == "bfloat16" else want):
        raise ValueError(f"{what}: {dtype} expected, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(shape)} expected, got {tuple(t.shape)}")


_int32 = _float32 = None  # torch's, once a tensor has been looked at


def _rows_held(t, ld, what, floats=False):
    """How many rows, ld entries apart, a tensor of int32 (or float32) holds
    (the kernels read them by its address); an address is taken as it is."""
    if t is None or isinstance(t, int):
        return 1 << 62
    global _int32, _float32
    if _int32 is None:
        import torch
        _int32, _float32 = torch.int32, torch.float32
    want = _float32 if floats else _int32
    if t.dtype != want:
        raise ValueError(f"{what}: {want} expected, got {t.dtype}")
    if t.is_contiguous() and (t.dim() != 2 or t.shape[0] != 1):
        return t.numel() // ld
    if t.dim() == 2 and (t.shape[0] == 1 or t.stride(0) == ld) and (t.shape[1] == 1 or t.stride(1) == 1):
        # (part of a wider one: its rows end where the storage does)
        return (t.untyped_storage().nbytes() // 4 - t.storage_offset()) // ld
    raise ValueError(f"{what}: adjacent entries, rows {ld} apart, expected")


def _expect_rows(t, rows, ld, what, floats=False):
    have = _rows_held(t, ld, what, floats)
    if have < rows:
        raise ValueError(f"{what}: holds {have} rows of {ld}, {rows} needed")


def _expect_table(rope: Rope, table):
    _expect_rows(table, rope.n_pos * rope.rotary_dim, 1, "table", True)


def _dims_held(dims, **tensors):
    """What a cfg has to have (the batch first), or, where a tensor (given
    with its entries a sequence) holds fewer sequences, what none has."""
    for what, (t, ld) in tensors.items():
        have = _rows_held(t, max(1, int(ld)), what)
        if have < dims[0]:
            return dims + (f"{what} for {have} sequences only",)
    return dims


def _same_shape(cfg: Cfg, io, where):
    if io._dims != (cfg.batch, cfg.n_kv_heads, cfg.head_dim):
        raise ValueError(f"{where}: built for (batch, n_kv_heads, head_dim) = {io._dims}, "
                         f"cfg has {(cfg.batch, cfg.n_kv_heads, cfg.head_dim)}")


def _as_rows(t) -> Rows:
    return t if isinstance(t, Rows) else rows_of(t)


def epikv_rope_table(rope: Rope, table, stream=None):
    if not isinstance(table, int):
        have = table.numel() * table.element_size()
        if have < rope_table_bytes(rope):
            raise ValueError(f"table holds {have} bytes, {rope_table_bytes(rope)} needed")
    _check(lib().epikv_rope_table(ctypes.byref(rope), _ptr(table), _stream(stream)),
           "epikv_rope_table")


def epikv_rope(rope: Rope, table, dtype, batch, chunk, n_heads, head_dim, x,
               y, positions, ld_pos=0, transpose=False, seq_status=None,
               stream=None):
    """x and y: tensors [batch][chunk][n_heads][head_dim], or Rows."""
    # (this call's time is the host's for a token a sequence: no more than needed)
    if x.__class__ is Rows and y.__class__ is Rows:
        xr, yr = x, y
    else:
        for t, what in ((x, "x"), (y, "y")):
            _expect(t, "float32" if dtype == DTYPE_FP32 else "bfloat16",
                    (batch, chunk, n_heads, head_dim), what)
        xr, yr = _as_rows(x), _as_rows(y)
    try:
        enough = (table.nbytes >= 4 * rope.n_pos * rope.rotary_dim and table.dtype is _float32
                  and positions.nbytes >= 4 * batch * (ld_pos or 1) and positions.dtype is _int32
                  and table.is_contiguous() and positions.is_contiguous())
    except AttributeError:  # (addresses)
        enough = False
    if enough:
        table, positions = table.data_ptr(), positions.data_ptr()
    else:
        _expect_table(rope, table)
        _expect_rows(positions, batch, ld_pos or 1, "positions")
        table, positions = _ptr(table), _ptr(positions)
    if seq_status is not None:
        _expect_rows(seq_status, batch, 1, "seq_status")
        seq_status = _ptr(seq_status)
    status = (_lib or lib()).epikv_rope(
        rope, table, int(dtype), int(batch), int(chunk), int(n_heads), int(head_dim), xr, yr, positions,
        int(ld_pos), int(transpose), seq_status, _stream(stream))
    if status != EPIKV_OK:
        _check(status, "epikv_rope")


def epikv_rope_axes_table(rope: Rope, axes: Axes, table, stream=None):
    if not isinstance(table, int):
        have = table.numel() * table.element_size()
        if have < rope_table_bytes(rope):
            raise ValueError(f"table holds {have} bytes, {rope_table_bytes(rope)} needed")
    _check(lib().epikv_rope_axes_table(ctypes.byref(rope), ctypes.byref(axes), _ptr(table), _stream(stream)),
           "epikv_rope_axes_table")


def epikv_rope_axes(rope: Rope, axes: Axes, table, dtype, batch, chunk, n_heads,
                    head_dim, x, y, positions, ld_pos=0, transpose=False,
                    seq_status=None, stream=None):
    """epikv_rope with positions [batch][n_axes], or [batch][n_axes][ld_pos]."""
    # (as short as epikv_rope, for the same reason)
    per_seq = max(1, axes.n_axes) * (ld_pos or 1)
    if x.__class__ is Rows and y.__class__ is Rows:
        xr, yr = x, y
    else:
        for t, what in ((x, "x"), (y, "y")):
            _expect(t, "float32" if dtype == DTYPE_FP32 else "bfloat16",
                    (batch, chunk, n_heads, head_dim), what)
        xr, yr = _as_rows(x), _as_rows(y)
    try:
        enough = (table.nbytes >= 4 * rope.n_pos * rope.rotary_dim and table.dtype is _float32
                  and positions.nbytes >= 4 * batch * per_seq and positions.dtype is _int32
                  and table.is_contiguous() and positions.is_contiguous())
    except AttributeError:  # (addresses)
        enough = False
    if enough:
        table, positions = table.data_ptr(), positions.data_ptr()
    else:
        _expect_table(rope, table)
        _expect_rows(positions, batch, per_seq, "positions")
        table, positions = _ptr(table), _ptr(positions)
    if seq_status is not None:
        _expect_rows(seq_status, batch, 1, "seq_status")
        seq_status = _ptr(seq_status)
    status = (_lib or lib()).epikv_rope_axes(
        rope, axes, table, int(dtype), int(batch), int(chunk), int(n_heads), int(head_dim), xr, yr, positions,
        int(ld_pos), int(transpose), seq_status, _stream(stream))
    if status != EPIKV_OK:
        _check(status, "epikv_rope_axes")


def make_append_io(chunk, pool: Pool, layer, page_table, ld_pt, n_cached, k, v,
                   n_new=None, rope: Rope | None = None, table=None,
                   positions=None, ld_pos=0, q=None, q_out=None, pos=None,
                   ld_s=0, seq_status=None, axes: Axes | None = None, ids=None,
                   ld_ids=0) -> AppendIO:
    """Build the epikv_append_io struct; k, v, q and q_out are tensors
    [B][chunk][heads][head_dim].  The object keeps what it was built from.
    With axes (and ids, where pos is given) it is for epikv_append_axes."""
    for t, like, what in ((v, k, "v"), (q_out, q, "q_out")):
        if t is not None:
            _expect(t, "bfloat16", like.shape, what)
    _expect(k, "bfloat16", (k.shape[0], int(chunk)) + tuple(k.shape[2:]), "k")
    if q is not None:
        _expect(q, "bfloat16", (k.shape[0], int(chunk), q.shape[2], k.shape[3]), "q")
    if rope is not None:
        _expect_table(rope, table)
    io = AppendIO()
    io._dims = _dims_held((k.shape[0], k.shape[2], k.shape[3]), page_table=(page_table, ld_pt),
                          n_cached=(n_cached, 1), n_new=(n_new, 1),
                          positions=(positions, max(1, int(ld_pos)) * (max(1, axes.n_axes) if axes else 1)),
                          pos=(pos, ld_s), seq_status=(seq_status, 1), ids=(ids, ld_ids))
    io._keepalive = [page_table, n_cached, n_new, k, v, rope, table, positions,
                     q, q_out, pos, seq_status, axes, ids]
    io._axes = None if axes is None else (axes, _ptr(ids), int(ld_ids))
    io.chunk, io.layer, io.pool = int(chunk), int(layer), pool
    io.page_table, io.ld_pt = _ptr(page_table), int(ld_pt)
    io.n_cached, io.n_new = _ptr(n_cached), _ptr(n_new)
    io.k, io.v = rows_of(k), rows_of(v)
    io.rope = ctypes.pointer(rope) if rope is not None else None
    io.rope_table = _ptr(table)
    io.positions, io.ld_pos = _ptr(positions), int(ld_pos)
    io.n_heads = int(q.shape[2]) if q is not None else 0
    io.q, io.q_out = rows_of(q), rows_of(q_out)
    io.pos, io.ld_s, io.seq_status = _ptr(pos), int(ld_s), _ptr(seq_status)
    return io


def epikv_append(cfg: Cfg, io: AppendIO, stream=None):
    _same_shape(cfg, io, "epikv_append")
    if io._axes is not None:
        raise ValueError("epikv_append: built with axes, for epikv_append_axes")
    _check(lib().epikv_append(ctypes.byref(cfg), ctypes.byref(io),
                              _stream(stream)), "epikv_append")


def epikv_append_axes(cfg: Cfg, io: AppendIO, stream=None):
    """io: make_append_io with axes (and ids)."""
    _same_shape(cfg, io, "epikv_append_axes")
    if io._axes is None:
        raise ValueError("epikv_append_axes: built without axes, for epikv_append")
    axes, ids, ld_ids = io._axes
    _check(lib().epikv_append_axes(ctypes.byref(cfg), ctypes.byref(io), ctypes.byref(axes), ids, ld_ids,
                                   _stream(stream)), "epikv_append_axes")


def make_read_io(chunk, pool: Pool, layer, page_table, ld_pt, first, k=None,
                 v=None, seq_status=None) -> ReadIO:
    like = v if k is None else k
    for t, what in ((k, "k"), (v, "v")):
        _expect(t, "bfloat16", (like.shape[0], int(chunk)) + tuple(like.shape[2:]), what)
    io = ReadIO()
    io._dims = _dims_held((like.shape[0], like.shape[2], like.shape[3]), page_table=(page_table, ld_pt),
                          first=(first, 1), seq_status=(seq_status, 1))
    io._keepalive = [page_table, first, k, v, seq_status]
    io.chunk, io.layer, io.pool = int(chunk), int(layer), pool
    io.page_table, io.ld_pt, io.first = _ptr(page_table), int(ld_pt), _ptr(first)
    io.k, io.v, io.seq_status = rows_of(k), rows_of(v), _ptr(seq_status)
    return io


def epikv_read(cfg: Cfg, io: ReadIO, stream=None):
    _same_shape(cfg, io, "epikv_read")
    _check(lib().epikv_read(ctypes.byref(cfg), ctypes.byref(io),
                            _stream(stream)), "epikv_read")


def make_attend_io(chunk, pool: Pool, layer, page_table, ld_pt, n_cached, q, out,
                   n_new=None, lse=None, scale=0.0, seq_status=None,
                   workspace=None, workspace_bytes_=0) -> AttendIO:
    """Build the epikv_attend_io struct; q and out are tensors
    [B][chunk][n_heads][head_dim], lse float32 [B][n_heads][chunk]."""
    B, _, n_heads, d = q.shape
    for t, what in ((q, "q"), (out, "out")):
        _expect(t, "bfloat16", (B, int(chunk), n_heads, d), what)
    if lse is not None:
        _expect(lse, "float32", (B, n_heads, int(chunk)), "lse")
        if not lse.is_contiguous():
            raise ValueError("lse must be contiguous")
    io = AttendIO()
    io._dims = _dims_held((B, d), page_table=(page_table, ld_pt), n_cached=(n_cached, 1), n_new=(n_new, 1),
                          seq_status=(seq_status, 1))
    io._keepalive = [page_table, n_cached, n_new, q, out, lse, seq_status, workspace]
    io.chunk, io.layer, io.pool = int(chunk), int(layer), pool
    io.page_table, io.ld_pt = _ptr(page_table), int(ld_pt)
    io.n_cached, io.n_new, io.n_heads = _ptr(n_cached), _ptr(n_new), int(n_heads)
    io.q, io.out, io.lse = rows_of(q), rows_of(out), _ptr(lse)
    io.scale, io.seq_status = float(scale), _ptr(seq_status)
    io.workspace = _ws(workspace, workspace_bytes_)
    io.workspace_bytes = int(workspace_bytes_)
    return io


def _same_attend(cfg: Cfg, io: AttendIO, where):
    if io._dims != (cfg.batch, cfg.head_dim):
        raise ValueError(f"{where}: built for (batch, head_dim) = {io._dims}, "
                         f"cfg has {(cfg.batch, cfg.head_dim)}")


def epikv_attend(cfg: Cfg, io: AttendIO, stream=None):
    _same_attend(cfg, io, "epikv_attend")
    _check(lib().epikv_attend(ctypes.byref(cfg), ctypes.byref(io),
                              _stream(stream)), "epikv_attend")


def make_weigh_io(weights, ld_s, old=None, keep_old=1.0, keep_new=0.0, gain=1.0,
                  watch=0) -> WeighIO:
    """Build the epikv_weigh_io struct; weights and old are float32
    [batch][ld_s].  old may be weights itself: the sums go on in place."""
    io = WeighIO()
    io._held = min(_rows_held(t, max(1, int(ld_s)), what, True) for t, what in ((weights, "weights"), (old, "old")))
    io._keepalive = [weights, old]
    io.old, io.weights, io.ld_s = _ptr(old), _ptr(weights), int(ld_s)
    io.keep_old, io.keep_new, io.gain = float(keep_old), float(keep_new), float(gain)
    io.watch = int(watch)
    return io


def epikv_attend_weigh(cfg: Cfg, io: AttendIO, weigh: WeighIO, stream=None):
    _same_attend(cfg, io, "epikv_attend_weigh")
    if weigh._held < cfg.batch:
        raise ValueError(f"epikv_attend_weigh: sums for {weigh._held} sequences, cfg has {cfg.batch}")
    _check(lib().epikv_attend_weigh(ctypes.byref(cfg), ctypes.byref(io), ctypes.byref(weigh),
                                    _stream(stream)), "epikv_attend_weigh")


# ---------------------------------------------------------------------------
# State buffer views (the documented layout of include/epikv.h)
# ---------------------------------------------------------------------------
def n_sig(cfg: Cfg) -> int:
    return cfg.n_band_a + cfg.n_band_b if cfg.signal == SIGNAL_HS else 1


def state_sections(cfg: Cfg, state):
    """Typed views of a uint8 state tensor (CPU or device):
    dict(n_tok [B] int32, ring [B][n_sig][w-1] float32, ema [B][n_sig],
         h_prev [B][n_band][D] int16 (HS), range [2][B][L][2][H][d] float32
         (lag-normalised KV signals))."""
    import torch
    off = state_layout(cfg)
    B, w = cfg.batch, cfg.window
    out = {}
    out["n_tok"] = state[off[0]:off[0] + 4 * B].view(torch.int32)
    nr = B * n_sig(cfg) * (w - 1)
    out["ring"] = state[off[1]:off[1] + 4 * nr].view(torch.float32).view(
        B, n_sig(cfg), w - 1)
    if cfg.signal == SIGNAL_HS:
        nb = cfg.n_band_a + cfg.n_band_b
        nh = B * nb * cfg.hidden
        out["h_prev"] = state[off[2]:off[2] + 2 * nh].view(torch.int16).view(
            B, nb, cfg.hidden)
    elif cfg.signal in (SIGNAL_LAGKV, SIGNAL_LAGKV_KEY):
        shp = (2, B, cfg.n_layers, 2, cfg.n_kv_heads, cfg.head_dim)
        n = 1
        for s in shp:
            n *= s
        out["range"] = state[off[3]:off[3] + 4 * n].view(torch.float32).view(
            *shp)
    ne = B * n_sig(cfg)
    out["ema"] = state[off[4]:off[4] + 4 * ne].view(torch.float32).view(
        B, n_sig(cfg))
    return out
