"""ctypes binding of ``libwino.so`` (declared in ``include/wino.h``).

Argument marshalling only: every function forwards to the C entry point of
the same name, passing device pointers (``torch.Tensor.data_ptr()`` or raw
integers), sizes and a ``cudaStream_t`` handle.  All computation happens in
the library's CUDA kernels.  If the library has not been built, loading it
raises ``RuntimeError``; there is no fallback.
"""
from __future__ import annotations

import ctypes as C
from pathlib import Path

_LIB_PATH = Path(__file__).resolve().parent / "_build" / "libwino.so"
_lib = None

WINO_OK = 0
WINO_ERR_ARG = -1
WINO_ERR_SHAPE = -2
WINO_ERR_WORKSPACE = -3
WINO_ERR_CUDA = -4
WINO_ERR_MAX_STEPS = -5
WINO_ERR_DEVICE_TIMEOUT = -6
WINO_ERR_UNSUPPORTED = -7

# per-position outcome codes written to `flags`
FLAG_NONE, FLAG_DRAFT, FLAG_DRAFT_FALLBACK, FLAG_REMASK, FLAG_DRAFT_IS_MASK, FLAG_DRAFT_TOP_M = 0, 1, 2, 3, 4, 5

# wino_params.options
WINO_OPT_FREEZE_FINISHED = 1
WINO_OPT_NO_SHADOW = 2
WINO_OPT_COMPACT = 4
WINO_OPT_W_PANELS = 8

EXPORTS = ("wino_workspace_size", "wino_workspace_size_step", "wino_score_rows", "wino_draft_verify", "wino_step",
           "wino_step_static_scratch", "wino_read_device_status", "wino_profile_begin", "wino_profile_end",
           "wino_selftest_wait_timeout", "wino_status_string", "wino_version", "wino_decode", "wino_timeline_begin",
           "wino_timeline_end", "wino_score_plan", "wino_score_plan_host", "wino_score_launch", "wino_lm_head_panels",
           "wino_rope_frequencies", "wino_rope_append", "wino_attend_workspace_size", "wino_attend",
           "wino_norm_rope_append", "wino_cache_read", "wino_attend_scaled")

# wino_kv_batch.dtype, wino_kv_batch.mask, scalings of wino_rope_frequencies
WINO_BF16, WINO_FP16 = 0, 1
WINO_CACHE_E4M3 = 16
WINO_MASK_FULL, WINO_MASK_CAUSAL, WINO_MASK_SHADOW = 0, 1, 2
ROPE_SCALINGS = {"none": 0, "linear": 1, "parts": 2}

# bytes of status words at the start of a workspace: all that wino_rope_append uses of one
STATUS_BYTES = 256

# 64-bit words per CTA in a score-kernel timeline (wino_timeline_begin)
TIMELINE_WORDS = 8

# size of the fixed device array behind wino_step_static_scratch
WINO_STATIC_SCRATCH_BYTES = 16 << 20


class WinoError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {wino_status_string(status)} ({status})")


class WinoParams(C.Structure):
    _fields_ = [("tau1", C.c_float), ("tau2", C.c_float), ("mask_id", C.c_int32), ("n_seq", C.c_int32),
                ("seq_len", C.c_int32), ("blk_start", C.c_int32), ("blk_len", C.c_int32),
                ("max_steps", C.c_int32), ("options", C.c_int32), ("step_index", C.c_int32),
                ("last_change", C.c_void_p), ("draft_m", C.c_int32), ("active_seq", C.c_void_p),
                ("n_active", C.c_int32)]


class WinoBlockStats(C.Structure):
    _fields_ = [("steps", C.c_int32), ("drafted", C.c_int32), ("remasked", C.c_int32), ("fallback", C.c_int32),
                ("seq_steps", C.c_int32)]


class WinoHeads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class WinoKvBatch(C.Structure):
    """wino_kv_batch; ``make_kv_batch`` makes one and keeps its tensors alive."""
    _fields_ = [("n_seq", C.c_int32), ("n_rows", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("mask", C.c_int32), ("page_size", C.c_int32),
                ("n_pages", C.c_int32), ("table_width", C.c_int32), ("q_start", C.c_void_p), ("q_len", C.c_void_p),
                ("kv_len", C.c_void_p), ("new_slot", C.c_void_p), ("page_table", C.c_void_p),
                ("k_cache", C.c_void_p), ("v_cache", C.c_void_p), ("page_stride", C.c_int64),
                ("slot_stride", C.c_int64), ("head_stride", C.c_int64)]


class WinoRope(C.Structure):
    """wino_rope; ``make_rope`` makes one and keeps its tensors alive."""
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("factor", C.c_float), ("freq", C.c_void_p),
                ("positions", C.c_void_p)]


class WinoKvScales(C.Structure):
    """wino_kv_scales; ``make_kv_batch`` makes one beside the batch of an 8-bit cache."""
    _fields_ = [("k_scale", C.c_void_p), ("v_scale", C.c_void_p)]


class WinoHeadNorm(C.Structure):
    """wino_head_norm; ``make_head_norm`` makes one and keeps its tensors alive."""
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("q_head_stride", C.c_int64),
                ("k_head_stride", C.c_int64), ("eps", C.c_float), ("offset", C.c_float)]


class WinoRopeAxes(C.Structure):
    """wino_rope_axes; ``make_rope_axes`` makes one and keeps its tensors alive."""
    _fields_ = [("n_axes", C.c_int32), ("axis", C.c_void_p), ("positions", C.c_void_p), ("axis_stride", C.c_int64)]


# const uint16_t *(*)(void *user, int32_t step, int32_t blk_start)
HIDDEN_FN = C.CFUNCTYPE(C.c_void_p, C.c_void_p, C.c_int32, C.c_int32)


def library_path() -> Path:
    return _LIB_PATH


def lib() -> C.CDLL:
    """Load libwino.so (built in-tree by ``__graft_entry__.build()``)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with paper_2605_16941_gb300.build.build()")
        L = C.CDLL(str(_LIB_PATH))
        i64, vp, sz = C.c_int64, C.c_void_p, C.c_size_t
        L.wino_workspace_size.restype = C.c_int
        L.wino_workspace_size.argtypes = [i64, i64, i64, C.POINTER(sz)]
        L.wino_workspace_size_step.restype = C.c_int
        L.wino_workspace_size_step.argtypes = [C.POINTER(WinoParams), i64, i64, C.POINTER(sz)]
        L.wino_score_rows.restype = C.c_int
        L.wino_score_rows.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        L.wino_draft_verify.restype = C.c_int
        L.wino_draft_verify.argtypes = [vp, vp, vp, vp, C.POINTER(WinoParams), vp, vp, vp]
        L.wino_step.restype = C.c_int
        L.wino_step.argtypes = [vp, vp, i64, i64, vp, C.POINTER(WinoParams), vp, vp, vp, sz, vp]
        heads, batch = C.POINTER(WinoHeads), C.POINTER(WinoKvBatch)
        L.wino_rope_frequencies.restype = C.c_int
        L.wino_rope_frequencies.argtypes = [C.c_int32, C.c_double, C.c_int32, C.c_double, i64, C.POINTER(C.c_double),
                                            C.POINTER(C.c_float)]
        L.wino_rope_append.restype = C.c_int
        L.wino_rope_append.argtypes = [heads, heads, heads, heads, batch, C.POINTER(WinoRope), vp, vp]
        L.wino_attend_workspace_size.restype = C.c_int
        L.wino_attend_workspace_size.argtypes = [batch, C.POINTER(sz)]
        L.wino_attend.restype = C.c_int
        L.wino_attend.argtypes = [heads, heads, C.c_float, batch, vp, sz, vp]
        scales = C.POINTER(WinoKvScales)
        L.wino_norm_rope_append.restype = C.c_int
        L.wino_norm_rope_append.argtypes = [heads, heads, heads, heads, batch, C.POINTER(WinoRope),
                                            C.POINTER(WinoRopeAxes), C.POINTER(WinoHeadNorm), scales, vp, vp]
        L.wino_cache_read.restype = C.c_int
        L.wino_cache_read.argtypes = [heads, heads, batch, scales, vp, vp]
        L.wino_attend_scaled.restype = C.c_int
        L.wino_attend_scaled.argtypes = [heads, heads, C.c_float, batch, scales, vp, sz, vp]
        L.wino_lm_head_panels.restype = C.c_int
        L.wino_lm_head_panels.argtypes = [vp, i64, i64, vp, vp]
        L.wino_step_static_scratch.restype = C.c_int
        L.wino_step_static_scratch.argtypes = [vp, vp, i64, i64, vp, C.POINTER(WinoParams), vp, vp, vp]
        L.wino_read_device_status.restype = C.c_int
        L.wino_read_device_status.argtypes = [vp, vp, C.POINTER(C.c_int)]
        L.wino_profile_begin.restype = C.c_int
        L.wino_profile_begin.argtypes = [C.c_int]
        L.wino_profile_end.restype = C.c_int
        L.wino_profile_end.argtypes = [C.POINTER(C.c_double), C.POINTER(C.c_int)]
        L.wino_score_plan_host.restype = C.c_int
        L.wino_score_plan_host.argtypes = [i64, i64, i64, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
        L.wino_score_launch.restype = C.c_int
        L.wino_score_launch.argtypes = [i64, i64, i64, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
        L.wino_score_plan.restype = C.c_int
        L.wino_score_plan.argtypes = [i64, i64, i64, C.POINTER(C.c_int32)]
        L.wino_timeline_begin.restype = C.c_int
        L.wino_timeline_begin.argtypes = [vp, i64, i64]
        L.wino_timeline_end.restype = C.c_int
        L.wino_timeline_end.argtypes = [C.POINTER(i64)]
        L.wino_selftest_wait_timeout.restype = C.c_int
        L.wino_selftest_wait_timeout.argtypes = [vp, i64, vp]
        L.wino_status_string.restype = C.c_char_p
        L.wino_status_string.argtypes = [C.c_int]
        L.wino_version.restype = C.c_int
        L.wino_version.argtypes = []
        L.wino_decode.restype = C.c_int
        L.wino_decode.argtypes = [vp, i64, i64, vp, C.POINTER(WinoParams), C.c_int32, C.c_int32, C.c_int32,
                                  HIDDEN_FN, vp, vp, vp, vp, vp, vp, vp, sz, vp, C.POINTER(WinoBlockStats),
                                  C.POINTER(C.c_int32)]
        _lib = L
    return _lib


def _ptr(x) -> int | None:
    if x is None or isinstance(x, int):
        return x
    return x.data_ptr()


_raw_stream = None  # () -> handle of PyTorch's current stream on the current device


def _find_raw_stream():
    """torch.cuda.current_stream() builds a Stream object for the handle, which takes 3 us of a step whose kernels take
    9 us; PyTorch's raw query takes 0.2 us."""
    global _raw_stream
    import torch
    torch.cuda.current_stream()  # initialises CUDA, or raises what it raises without a device
    device = getattr(torch._C, "_cuda_getDevice", None)
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if device is not None and raw is not None:
        _raw_stream = lambda: raw(device())  # noqa: E731
    else:
        _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    return _raw_stream


def _stream(stream) -> int | None:
    if stream is None:
        return (_raw_stream or _find_raw_stream())()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int, where: str) -> None:
    if status != WINO_OK:
        raise WinoError(status, where)


def _nbytes(t) -> int:
    return t.numel() * t.element_size()


def wino_status_string(status: int) -> str:
    return lib().wino_status_string(int(status)).decode()


def wino_version() -> int:
    return lib().wino_version()


def wino_workspace_size(N: int, d: int, V: int) -> int:
    out = C.c_size_t(0)
    _check(lib().wino_workspace_size(N, d, V, C.byref(out)), "wino_workspace_size")
    return out.value


def wino_workspace_size_step(params: WinoParams, d: int, V: int) -> int:
    out = C.c_size_t(0)
    _check(lib().wino_workspace_size_step(C.byref(params), d, V, C.byref(out)), "wino_workspace_size_step")
    return out.value


def step_workspace(params: WinoParams, d: int, V: int, device=None):
    """A zeroed uint8 device tensor of wino_workspace_size_step bytes (allocated by PyTorch)."""
    import torch
    return torch.zeros(wino_workspace_size_step(params, d, V), dtype=torch.uint8, device=device or "cuda")


def workspace(N: int, d: int, V: int, device=None):
    """A zeroed uint8 device tensor of wino_workspace_size(N, d, V) bytes (allocated by PyTorch)."""
    import torch
    return torch.zeros(wino_workspace_size(N, d, V), dtype=torch.uint8, device=device or "cuda")


def make_params(tau1: float, tau2: float, mask_id: int, n_seq: int, seq_len: int, blk_start: int, blk_len: int,
                max_steps: int = 4096, freeze_finished: bool = False, step_index: int = 0,
                last_change=None, no_shadow: bool = False, compact: bool = False, draft_m: int = 0,
                active_seq=None, n_active: int | None = None, w_panels: bool = False) -> WinoParams:
    """wino_params; ``draft_m`` > 0 selects fixed-M drafting (naive parallel sampling, Sec. 3);
    ``active_seq`` (device int32) lists the sequences a wino_step scores and updates (default: all);
    ``w_panels``: the W passed to the step is the panel copy of ``wino_lm_head_panels``."""
    opts = ((WINO_OPT_FREEZE_FINISHED if freeze_finished else 0) | (WINO_OPT_NO_SHADOW if no_shadow else 0) |
            (WINO_OPT_COMPACT if compact else 0) | (WINO_OPT_W_PANELS if w_panels else 0))
    if active_seq is not None and n_active is None:
        n_active = int(active_seq.numel())
    return WinoParams(tau1, tau2, mask_id, n_seq, seq_len, blk_start, blk_len, max_steps, opts, step_index,
                      _ptr(last_change), draft_m, _ptr(active_seq), n_active or 0)


def wino_score_rows(H, W, target, argmax, pmax, ptarget, ws, stream=None, *, entropy=None, N: int | None = None,
                    d: int | None = None, V: int | None = None) -> None:
    """Fused LM-head + full-vocabulary softmax statistics (and, given ``entropy``, H(p) per row);
    shapes default to H.shape / W.shape."""
    N = H.size(0) if N is None else N
    d = H.size(1) if d is None else d
    V = W.size(0) if V is None else V
    ws_bytes = _nbytes(ws)
    _check(lib().wino_score_rows(_ptr(H), _ptr(W), N, d, V, _ptr(target), _ptr(argmax), _ptr(pmax), _ptr(ptarget),
                                 _ptr(entropy), _ptr(ws), ws_bytes, _stream(stream)), "wino_score_rows")


def wino_draft_verify(tokens, argmax, pmax, ptarget, params: WinoParams, counts, flags=None, stream=None) -> None:
    """Eq. 4 in place on ``tokens`` from per-row statistics."""
    _check(lib().wino_draft_verify(_ptr(tokens), _ptr(argmax), _ptr(pmax), _ptr(ptarget), C.byref(params),
                                   _ptr(counts), _ptr(flags), _stream(stream)), "wino_draft_verify")


def _vocab(W, params: WinoParams) -> int:
    """V from W's shape: [V, d] row-major, or [d/64, V, 64] for a panel copy (WINO_OPT_W_PANELS)."""
    return W.size(1 if params.options & WINO_OPT_W_PANELS else 0)


def wino_lm_head_panels(W, Wp=None, stream=None):
    """The panel copy Wp[k][v][c] = W[v][64k + c] of a [V, d] bf16 LM head, as a [d/64, V, 64] tensor (written
    into ``Wp`` when given, else allocated by PyTorch); pass it as W with ``make_params(..., w_panels=True)``."""
    import torch
    V, d = int(W.shape[0]), int(W.shape[1])
    if Wp is None:
        Wp = torch.empty((d // 64, V, 64), dtype=W.dtype, device=W.device)
    _check(lib().wino_lm_head_panels(_ptr(W), d, V, _ptr(Wp), _stream(stream)), "wino_lm_head_panels")
    return Wp


def wino_step(H, W, tokens, params: WinoParams, counts, ws, flags=None, stream=None, *, d: int | None = None,
              V: int | None = None) -> None:
    """One whole WINO step in place on ``tokens``."""
    d = H.size(1) if d is None else d
    V = _vocab(W, params) if V is None else V
    ws_bytes = _nbytes(ws)
    _check(lib().wino_step(_ptr(H), _ptr(W), d, V, _ptr(tokens), C.byref(params), _ptr(counts), _ptr(flags),
                           _ptr(ws), ws_bytes, _stream(stream)), "wino_step")


def wino_step_static_scratch(H, W, tokens, params: WinoParams, counts, flags=None, stream=None, *,
                             d: int | None = None, V: int | None = None) -> None:
    """wino_step with the library's fixed device scratch instead of a caller workspace (allocates nothing)."""
    d = H.size(1) if d is None else d
    V = _vocab(W, params) if V is None else V
    _check(lib().wino_step_static_scratch(_ptr(H), _ptr(W), d, V, _ptr(tokens), C.byref(params), _ptr(counts),
                                          _ptr(flags), _stream(stream)), "wino_step_static_scratch")


def wino_decode(W, tokens, params: WinoParams, n_blocks: int, hidden, counts, counts_host, ws, flags=None,
                stream=None, *, flags_host=None, active_buf=None, first_block: int = 0, first_step: int = 0,
                d: int | None = None, V: int | None = None):
    """The library's decode loop (wino_decode).  ``hidden(k, blk_start)`` returns step k's device bf16
    hidden states (a tensor, kept alive until the next call); ``counts_host`` is a host int32 [n_seq, 3]
    tensor (pinned for speed); with ``flags`` and a host int8 ``flags_host`` the at-least-one drafts are
    counted too; with a device int32 [n_seq] ``active_buf`` only the sequences whose block still has a
    MASK are stepped.  Returns (status, per-block (steps, drafted, re-masked, at-least-one drafts,
    sequences stepped summed over the steps), next step index); the status is
    WINO_OK or the error that stopped the loop (an exception raised by ``hidden`` is re-raised)."""
    if params.options & WINO_OPT_W_PANELS:  # [d/64, V, 64]
        d = int(W.shape[0]) * 64 if d is None else d
    else:
        d = int(W.shape[1]) if d is None else d
    V = _vocab(W, params) if V is None else V
    held, failure = [None], []

    def cb(user, k, blk_start):
        try:
            H = hidden(int(k), int(blk_start))
            held[0] = H
            return _ptr(H)
        except BaseException as e:  # reported after the call: an exception cannot cross the C frame
            failure.append(e)
            return None

    fn = HIDDEN_FN(cb)
    stats = (WinoBlockStats * n_blocks)()
    nxt = C.c_int32(0)
    ws_bytes = _nbytes(ws)
    rc = lib().wino_decode(_ptr(W), d, V, _ptr(tokens), C.byref(params), n_blocks, first_block, first_step, fn,
                           None, _ptr(counts), _ptr(counts_host), _ptr(flags), _ptr(flags_host), _ptr(active_buf),
                           _ptr(ws), ws_bytes, _stream(stream),
                           stats, C.byref(nxt))
    if failure:
        raise failure[0]
    return rc, [(b.steps, b.drafted, b.remasked, b.fallback, b.seq_steps) for b in stats], nxt.value


_raw_device = None  # () -> index of PyTorch's current device


def _current_device() -> int:
    """torch.cuda.current_device() without its lazy-initialisation check (1 us of a call)."""
    global _raw_device
    if _raw_device is None:
        import torch
        torch.cuda.current_device()
        _raw_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return _raw_device()


def _require(ok: bool, where: str, status: int = WINO_ERR_ARG) -> None:
    if not ok:
        raise WinoError(status, where)


def make_kv_batch(k_cache, v_cache, page_table, q_start, q_len, kv_len, new_slot, *, n_rows: int, n_q_heads: int,
                  mask: int, k_scale=None, v_scale=None, dtype=None) -> WinoKvBatch:
    """wino_kv_batch over a paged cache.  ``k_cache`` and ``v_cache`` are [n_pages, page_size, n_kv_heads, head_dim]
    views of one layout (a [pages, heads, slots, dim] cache is given as ``cache.transpose(1, 2)``), bfloat16, float16
    or 16-bit integers that hold bfloat16; ``page_table`` [n_seq, width] and the four length and slot arrays [n_seq]
    are contiguous int32 on the same device.  An 8-bit cache is float8_e4m3fn (or uint8 that holds such codes), with
    ``k_scale`` and ``v_scale`` contiguous uint8 [n_pages, n_kv_heads, page_size] and ``dtype`` the rows' element type
    (bfloat16 by default).  The batch keeps the tensors alive."""
    import torch
    where = "make_kv_batch"
    ints = (page_table, q_start, q_len, kv_len, new_slot)
    scaled = k_scale is not None or v_scale is not None
    _require(k_cache.dim() == 4 and v_cache.shape == k_cache.shape and v_cache.dtype == k_cache.dtype and
             k_cache.element_size() == (1 if scaled else 2) and page_table.dim() == 2, where, WINO_ERR_SHAPE)
    n_pages, page_size, n_kv_heads, head_dim = k_cache.shape
    live = [i for i in range(4) if k_cache.shape[i] > 1]  # strides of single entries say nothing
    _require(all(k_cache.stride(i) == v_cache.stride(i) for i in live) and k_cache.stride(3) == 1, where,
             WINO_ERR_SHAPE)
    _require(all(t.dtype == torch.int32 and t.is_contiguous() and t.device == k_cache.device for t in ints) and
             v_cache.device == k_cache.device, where)
    n_seq = page_table.size(0)
    _require(all(t.numel() == n_seq for t in ints[1:]), where, WINO_ERR_SHAPE)
    elements, scales = k_cache.dtype, None
    if scaled:
        elements = torch.bfloat16 if dtype is None else dtype
        _require(k_cache.dtype in (torch.float8_e4m3fn, torch.uint8) and elements in (torch.bfloat16, torch.float16) and
                 all(t is not None and t.dtype == torch.uint8 and t.is_contiguous() and t.device == k_cache.device
                     for t in (k_scale, v_scale)), where)
        _require(k_scale.shape == v_scale.shape == (n_pages, n_kv_heads, page_size), where, WINO_ERR_SHAPE)
        scales = WinoKvScales(_ptr(k_scale), _ptr(v_scale))
        scales.tensors = (k_scale, v_scale)
    else:
        _require(dtype is None or dtype == elements, where)
    b = WinoKvBatch(n_seq, n_rows, n_q_heads, n_kv_heads, head_dim,
                    (WINO_FP16 if elements == torch.float16 else WINO_BF16) | (WINO_CACHE_E4M3 if scaled else 0), mask,
                    page_size, n_pages, page_table.size(1), _ptr(q_start), _ptr(q_len), _ptr(kv_len), _ptr(new_slot),
                    _ptr(page_table), _ptr(k_cache), _ptr(v_cache), k_cache.stride(0), k_cache.stride(1), k_cache.stride(2))
    b.tensors = (k_cache, v_cache, *ints)
    b.scales = scales
    # plain attributes: what the calls compare with, cheaper than the struct's fields
    b.q_shape, b.kv_shape = (n_rows, n_q_heads, head_dim), (n_rows, n_kv_heads, head_dim)
    b.q_weights, b.k_weights = ((None, (head_dim,), (h, head_dim)) for h in (n_q_heads, n_kv_heads))  # of norms
    b.elements, b.device = elements, k_cache.get_device()
    b.devices = {b.device}
    return b


def make_rope(freq, *, rot_dim: int, factor: float = 1.0, interleaved: bool = False, positions=None) -> WinoRope:
    """wino_rope; ``freq`` is a device float64 [rot_dim / 2] tensor (None for rot_dim = 0), ``positions`` device int32
    [n_rows] or None."""
    import torch
    if rot_dim == 0:
        freq = None
    _require(rot_dim == 0 or (freq is not None and freq.dtype == torch.float64 and freq.is_contiguous() and
                              freq.numel() == rot_dim // 2), "make_rope", WINO_ERR_SHAPE)
    _require(positions is None or (positions.dtype == torch.int32 and positions.is_contiguous()), "make_rope")
    r = WinoRope(rot_dim, int(interleaved), factor, _ptr(freq), _ptr(positions))
    r.tensors = (freq, positions)
    r.devices = {t.get_device() for t in r.tensors if t is not None}
    r.n_positions = None if positions is None else positions.numel()
    return r


def make_rope_axes(axis, positions) -> WinoRopeAxes:
    """wino_rope_axes: ``axis`` device uint8 [rot_dim / 2], the axis of each pair; ``positions`` device int32
    [n_axes, n_rows] (rows of a wider array will do)."""
    import torch
    where = "make_rope_axes"
    _require(positions.dim() == 2 and axis.dim() == 1, where, WINO_ERR_SHAPE)
    _require(axis.dtype == torch.uint8 and axis.is_contiguous() and positions.dtype == torch.int32 and
             (positions.size(1) == 1 or positions.stride(1) == 1) and axis.device == positions.device, where)
    a = WinoRopeAxes(positions.size(0), _ptr(axis), _ptr(positions), positions.stride(0))
    a.tensors = (axis, positions)
    a.device = positions.get_device()
    a.n_pairs, a.n_positions = axis.numel(), positions.size(1)
    return a


def make_head_norm(q_weight, k_weight, *, eps: float = 1e-6, offset: float = 0.0) -> WinoHeadNorm:
    """wino_head_norm: device weights of the element type, [head_dim] for all heads or [heads, head_dim], None for what is not
    normalised; ``offset`` 1 for weights that are kept as differences from 1."""
    where = "make_head_norm"
    given = [w for w in (q_weight, k_weight) if w is not None]
    _require(all(w.dim() in (1, 2) for w in given), where, WINO_ERR_SHAPE)
    _require(all(w.stride(-1) == 1 and w.element_size() == 2 for w in given) and
             len({(w.device, w.dtype) for w in given}) < 2, where)
    n = WinoHeadNorm(_ptr(q_weight), _ptr(k_weight), *(w.stride(0) if w is not None and w.dim() == 2 and w.size(0) > 1 else 0
                                                       for w in (q_weight, k_weight)), eps, offset)
    n.tensors = (q_weight, k_weight)
    n.devices = {w.get_device() for w in given}
    n.elements = given[0].dtype if given else None
    n.shapes = n.q_shape, n.k_shape = tuple(None if w is None else tuple(w.shape) for w in (q_weight, k_weight))
    return n


def wino_rope_frequencies(rot_dim: int, base: float, *, scaling: str = "none", factor: float = 1.0,
                          trained_len: int = 1):
    """(frequencies as a host float64 [rot_dim / 2] tensor, factor on the rotated values) for ``make_rope``.  ``scaling``: "none",
    "linear", or "parts" as in arXiv 2309.00071, with a ramp in turns from 1 to 32; for a checkpoint trained with another ramp
    or other bounds give ``make_rope`` frequencies and factor of its own."""
    import torch
    freq = torch.empty(max(rot_dim, 0) // 2, dtype=torch.float64)
    out = C.c_float(0)
    _check(lib().wino_rope_frequencies(rot_dim, base, ROPE_SCALINGS[scaling], factor, trained_len,
                                       C.cast(freq.data_ptr() or C.addressof(out), C.POINTER(C.c_double)),
                                       C.byref(out)), "wino_rope_frequencies")
    return freq, out.value


def _heads(t, b: WinoKvBatch, shape, where: str) -> WinoHeads:
    """A [n_rows, heads, head_dim] tensor as wino_heads."""
    if t.shape != shape:
        raise WinoError(WINO_ERR_SHAPE, where)
    row, head, one = t.stride()
    if one != 1 or t.dtype is not b.elements or t.get_device() != b.device:
        raise WinoError(WINO_ERR_ARG, where)
    return WinoHeads(t.data_ptr(), row, head)


def _append_args(q, k, v, batch: WinoKvBatch, rope: WinoRope, ws, q_out, where: str):
    """The heads of an append, checked together with what is common to both appends."""
    qh = qo = kh = vh = None
    if q is not None:
        qh = _heads(q, batch, batch.q_shape, where)
        qo = qh if q_out is None else _heads(q_out, batch, batch.q_shape, where)
    if k is not None:
        kh = _heads(k, batch, batch.kv_shape, where)
    if v is not None:
        vh = _heads(v, batch, batch.kv_shape, where)
    if rope.n_positions not in (None, batch.q_shape[0]):
        raise WinoError(WINO_ERR_SHAPE, where)
    if ws.numel() * ws.element_size() < STATUS_BYTES:
        raise WinoError(WINO_ERR_WORKSPACE, where)
    # the kernels run on the current device; wino_rope_frequencies' values are on the host
    if not rope.devices <= batch.devices or not batch.device == _current_device() == ws.get_device():
        raise WinoError(WINO_ERR_ARG, where)
    return qh, qo, kh, vh


def wino_rope_append(q, k, v, batch: WinoKvBatch, rope: WinoRope, ws, *, q_out=None, stream=None) -> None:
    """Rotate the rows' queries (into ``q_out``, or in place) and write their rotated keys and their values into the
    batch's cache.  ``q`` None: the cache alone; ``k`` and ``v`` None: the queries alone."""
    where = "wino_rope_append"
    qh, qo, kh, vh = _append_args(q, k, v, batch, rope, ws, q_out, where)
    status = lib().wino_rope_append(qh, qo, kh, vh, batch, rope, ws.data_ptr(), _stream(stream))
    if status != WINO_OK:
        raise WinoError(status, where)


def wino_norm_rope_append(q, k, v, batch: WinoKvBatch, rope: WinoRope, ws, *, norm: WinoHeadNorm | None = None,
                          axes: WinoRopeAxes | None = None, q_out=None, stream=None) -> None:
    """``wino_rope_append`` with per-head norms of queries and keys (``norm``), positions of several axes (``axes``, with a
    ``rope`` without positions), and into an 8-bit cache where ``batch`` has one."""
    where = "wino_norm_rope_append"
    qh, qo, kh, vh = _append_args(q, k, v, batch, rope, ws, q_out, where)
    if axes is not None:
        if axes.n_positions != batch.q_shape[0] or axes.n_pairs != rope.rot_dim // 2:
            raise WinoError(WINO_ERR_SHAPE, where)
        if axes.device != batch.device:
            raise WinoError(WINO_ERR_ARG, where)
    if norm is not None:
        if norm.q_shape not in batch.q_weights or norm.k_shape not in batch.k_weights:
            raise WinoError(WINO_ERR_SHAPE, where)
        if not norm.devices <= batch.devices or norm.elements not in (None, batch.elements):
            raise WinoError(WINO_ERR_ARG, where)
    status = lib().wino_norm_rope_append(qh, qo, kh, vh, batch, rope, axes, norm, batch.scales, ws.data_ptr(), _stream(stream))
    if status != WINO_OK:
        raise WinoError(status, where)


def wino_cache_read(k, v, batch: WinoKvBatch, ws, *, stream=None) -> None:
    """The batch's rows out of its cache, from the slots at which an append with the same batch stores them, into ``k`` and ``v``
    [n_rows, n_kv_heads, head_dim] (either may be None)."""
    where = "wino_cache_read"
    kh = None if k is None else _heads(k, batch, batch.kv_shape, where)
    vh = None if v is None else _heads(v, batch, batch.kv_shape, where)
    if ws.numel() * ws.element_size() < STATUS_BYTES:
        raise WinoError(WINO_ERR_WORKSPACE, where)
    if not batch.device == _current_device() == ws.get_device():
        raise WinoError(WINO_ERR_ARG, where)
    status = lib().wino_cache_read(kh, vh, batch, batch.scales, ws.data_ptr(), _stream(stream))
    if status != WINO_OK:
        raise WinoError(status, where)


def wino_attend_workspace_size(batch: WinoKvBatch) -> int:
    out = C.c_size_t(0)
    _check(lib().wino_attend_workspace_size(batch, C.byref(out)), "wino_attend_workspace_size")
    return out.value


def attend_workspace(batch: WinoKvBatch):
    """A zeroed uint8 device tensor of wino_attend_workspace_size bytes, beside the batch's cache."""
    import torch
    return torch.zeros(wino_attend_workspace_size(batch), dtype=torch.uint8, device=batch.tensors[0].device)


def append_workspace(device=None):
    """A zeroed uint8 device tensor of the status words, for wino_rope_append without a wino_attend behind it."""
    import torch
    return torch.zeros(STATUS_BYTES, dtype=torch.uint8, device=device or "cuda")


def _attend_args(q, out, batch: WinoKvBatch, ws, scale, where: str):
    qh, oh = _heads(q, batch, batch.q_shape, where), _heads(out, batch, batch.q_shape, where)
    if not batch.device == _current_device() == ws.get_device():  # the kernels run on the current device
        raise WinoError(WINO_ERR_ARG, where)
    return qh, oh, batch.q_shape[2] ** -0.5 if scale is None else scale


def wino_attend(q, out, batch: WinoKvBatch, ws, *, scale: float | None = None, stream=None) -> None:
    """Attention of the batch's rows over its cache, into ``out``; ``scale`` defaults to head_dim^-1/2."""
    where = "wino_attend"
    qh, oh, scale = _attend_args(q, out, batch, ws, scale, where)
    status = lib().wino_attend(qh, oh, scale, batch, ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream))
    if status != WINO_OK:
        raise WinoError(status, where)


def wino_attend_scaled(q, out, batch: WinoKvBatch, ws, *, scale: float | None = None, stream=None) -> None:
    """``wino_attend`` over an 8-bit cache."""
    where = "wino_attend_scaled"
    qh, oh, scale = _attend_args(q, out, batch, ws, scale, where)
    status = lib().wino_attend_scaled(qh, oh, scale, batch, batch.scales, ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream))
    if status != WINO_OK:
        raise WinoError(status, where)


def wino_read_device_status(ws, stream=None) -> int:
    """The status of a workspace's last call; of its paged-cache calls the first failure since this was last read, which is
    cleared."""
    out = C.c_int(0)
    _check(lib().wino_read_device_status(_ptr(ws), _stream(stream), C.byref(out)), "wino_read_device_status")
    return out.value


def wino_profile_begin(max_launches: int) -> None:
    _check(lib().wino_profile_begin(int(max_launches)), "wino_profile_begin")


def wino_profile_end() -> tuple[float, int]:
    """(summed score-kernel milliseconds, number of launches timed)."""
    ms, n = C.c_double(0), C.c_int(0)
    _check(lib().wino_profile_end(C.byref(ms), C.byref(n)), "wino_profile_end")
    return ms.value, n.value


def wino_score_plan(N: int, d: int, V: int) -> dict:
    """The row-block score kernel's work split for N rows over V entries on the current device."""
    out = (C.c_int32 * 8)()
    _check(lib().wino_score_plan(int(N), int(d), int(V), out), "wino_score_plan")
    return dict(zip(("bn", "n_vt", "n_mb", "n_groups", "G", "ctas", "two", "stages"), list(out)))


def wino_score_plan_host(N: int, d: int, V: int, sm_count: int = 152, max_pairs: int = 76) -> dict:
    """The row-block score kernel's work split for a device with sm_count SMs and max_pairs resident pairs (no device)."""
    out = (C.c_int32 * 10)()
    _check(lib().wino_score_plan_host(int(N), int(d), int(V), int(sm_count), int(max_pairs), out),
           "wino_score_plan_host")
    return dict(zip(("bn", "n_vt", "n_mb", "n_groups", "G", "ctas", "two", "stages", "stage_bytes",
                     "records_per_row"), list(out)))


def wino_score_launch(N: int, d: int, V: int, sm_count: int = 0, max_pairs: int = 0) -> dict:
    """The score kernel that runs for N rows (``kernel``: 0 row blocks in single tiles, 1 row blocks in passes,
    2 vocabulary-major) and its work split, on the current device or a described one."""
    out = (C.c_int32 * 14)()
    _check(lib().wino_score_launch(int(N), int(d), int(V), int(sm_count), int(max_pairs), out), "wino_score_launch")
    return dict(zip(("kernel", "bn", "n_vt", "n_groups", "G", "ctas", "records", "stages", "stage_bytes", "smem_bytes",
                     "hw0", "hw1", "slots", "split"), list(out)))


def wino_timeline_begin(buf, n_launches: int, ctas_per_launch: int) -> None:
    """Start recording per-CTA score-kernel stamps into the device uint64 tensor ``buf``
    (n_launches * ctas_per_launch * TIMELINE_WORDS words)."""
    _check(lib().wino_timeline_begin(_ptr(buf), int(n_launches), int(ctas_per_launch)), "wino_timeline_begin")


def wino_timeline_end() -> int:
    """Stop recording; returns the number of score launches counted."""
    n = C.c_int64(0)
    _check(lib().wino_timeline_end(C.byref(n)), "wino_timeline_end")
    return n.value


def wino_selftest_wait_timeout(status, limit_ns: int, stream=None) -> None:
    """Run the bounded-wait timeout self-test; ``status`` (device int32) receives the outcome."""
    _check(lib().wino_selftest_wait_timeout(_ptr(status), int(limit_ns), _stream(stream)),
           "wino_selftest_wait_timeout")
