"""Operators of sequence policies over episodes: Python binding of libqdseq.so
(the C ABI of include/qd_seq.h).

A sequence policy is told the wanted descriptor in its first tokens and reads
one token per step of an episode; it is fitted to the episodes of an archive's
elites, or rolled out in their place.  Its blocks are made of

  residual_norm        root-mean-square norm with the residual's addition
  window_attention     attention over a sliding window whose first tokens stay visible
  decay_attention      linear attention with a decay for each head

Each is differentiable under torch's autograd.  The calls below them are the
plain ones: `*_forward` and `*_backward` for programs that keep their own
tape, `residual_norm_fp8` for an 8-bit output, and `window_attention_step`
(with `window_cache` and `window_cache_fill`) and `decay_attention_step` for
rollouts, one token at a time.

Argument marshalling only: outputs and scratch memory are torch tensors, work
is enqueued on torch's current stream of the tensors' device, nothing waits for
the GPU, and there is no fallback.  Tensors are used on that stream alone; a
tensor made on another stream has to be synchronised with it first, as for any
torch operation.  Attention takes bfloat16 or float16 tensors whose rows start
at multiples of 16 bytes; others are copied first.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libqdseq.so")

ABI_VERSION = 1
OK, ERR_INVALID_ARG, ERR_WORKSPACE_TOO_SMALL, ERR_UNSUPPORTED, ERR_HIP = 0, 1, 2, 4, 5
F32, BF16, F16 = range(3)

# Every symbol include/qd_seq.h declares.
EXPORTS = ["qds_residual_norm", "qds_residual_norm_fp8", "qds_residual_norm_backward_workspace",
           "qds_residual_norm_backward", "qds_window_forward", "qds_window_backward_workspace",
           "qds_window_backward", "qds_window_step_workspace", "qds_window_step",
           "qds_window_cache_fill", "qds_decay_forward_workspace", "qds_decay_forward",
           "qds_decay_backward_workspace", "qds_decay_backward", "qds_decay_step",
           "qds_status_str"]


class QdsView(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64 * 3)]


class QdsNormConfig(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("dtype", C.c_int32), ("weight_dtype", C.c_int32),
                ("width", C.c_int32), ("rows", C.c_int64), ("eps", C.c_float), ("group", C.c_int32)]


class QdsWindowConfig(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("dtype", C.c_int32), ("batch", C.c_int32),
                ("length", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("dim", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32),
                ("scale", C.c_float)]


class QdsDecayConfig(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("dtype", C.c_int32), ("batch", C.c_int32),
                ("length", C.c_int32), ("heads", C.c_int32), ("dim_k", C.c_int32),
                ("dim_v", C.c_int32), ("scale", C.c_float)]


class SeqError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {lib().qds_status_str(status).decode()} (status {status})")


_lib = None


def lib():
    """The loaded libqdseq.so; raises if it was never built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        L = C.CDLL(LIB_PATH)
        P, U, I, V = C.c_void_p, C.c_uint64, C.c_int64, QdsView
        N, W, D = C.POINTER(QdsNormConfig), C.POINTER(QdsWindowConfig), C.POINTER(QdsDecayConfig)
        B = C.POINTER(C.c_uint64)
        L.qds_residual_norm.argtypes = [N, P, I, P, I, P, P, P, P, P]
        L.qds_residual_norm_fp8.argtypes = [N, P, I, P, I, P, P, P, P, P]
        L.qds_residual_norm_backward_workspace.argtypes = [N, B]
        L.qds_residual_norm_backward.argtypes = [N, P, I, P, I, P, I, P, P, P, P, P, U, P]
        L.qds_window_forward.argtypes = [W, V, V, V, P, V, P, P]
        L.qds_window_backward_workspace.argtypes = [W, B]
        L.qds_window_backward.argtypes = [W, V, V, V, V, V, P, P, V, V, V, P, U, P]
        L.qds_window_step_workspace.argtypes = [W, B]
        L.qds_window_step.argtypes = [W, V, V, V, P, P, P, V, P, U, P]
        L.qds_window_cache_fill.argtypes = [W, V, V, P, P, P, P]
        L.qds_decay_forward_workspace.argtypes = [D, B]
        L.qds_decay_forward.argtypes = [D, V, V, V, P, P, P, V, P, P, U, P]
        L.qds_decay_backward_workspace.argtypes = [D, B]
        L.qds_decay_backward.argtypes = [D, V, V, V, V, P, P, P, P, V, V, V, P, P, U, P]
        L.qds_decay_step.argtypes = [D, V, V, V, P, P, V, P, P]
        L.qds_status_str.argtypes = [C.c_int]
        L.qds_status_str.restype = C.c_char_p
        for name in EXPORTS[:-1]:
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _check(status: int, what: str):
    if status != OK:
        raise SeqError(status, what)


# ---------------------------------------------------------------------------
# Marshalling
# ---------------------------------------------------------------------------
_CODES = {}


def _codes():
    import torch
    if not _CODES:
        _CODES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    return _CODES


def _need(cond, message):
    if not cond:
        raise ValueError(message)


def _code(t, name):
    code = _codes().get(t.dtype)
    _need(code is not None, f"{name}: float32, bfloat16 or float16, not {t.dtype}")
    return code


def _like(name, t, ref, shape=None, dtype=None):
    """Checks a tensor's device, type and shape against those of `ref`."""
    _need(t.device == ref.device, f"{name} is on {t.device}, not on {ref.device}")
    _need(t.dtype == (dtype or ref.dtype), f"{name} is {t.dtype}, not {dtype or ref.dtype}")
    if shape is not None:
        _need(tuple(t.shape) == tuple(shape), f"{name} is {tuple(t.shape)}, not {tuple(shape)}")


def _on_gpu(t, name):
    if t.device.type != "cuda":
        raise RuntimeError(f"{name}: libqdseq needs tensors on a GPU, not on {t.device}")


def _rows(t):
    """`t` with contiguous, 16-byte aligned rows: itself, or a copy."""
    if t.stride(-1) == 1 and t.data_ptr() % 16 == 0 and not any(s % 8 for s in t.stride()[:-1]):
        return t
    import torch
    return t.clone(memory_format=torch.contiguous_format)


def _view(t):
    """A [batch, rows, heads, dim] or [batch, heads, dim] tensor as a qds_view."""
    s = t.stride()
    return QdsView(t.data_ptr(), (C.c_int64 * 3)(s[0], s[1] if len(s) == 4 else 0, s[-2]))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(t):
    import torch
    return torch.cuda.current_stream(t.device).cuda_stream


class _on:
    """The tensors' device as the current one (cheap where it already is)."""

    def __init__(self, t):
        import torch
        index = t.device.index
        self.guard = None if torch.cuda.current_device() == index else torch.cuda.device(index)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _workspace(query, cfg, ref, what):
    """Scratch memory of the size that `query` gives; torch's allocator keeps it
    from other work on this stream until the call's work is done."""
    import torch
    n = C.c_uint64()
    _check(query(C.byref(cfg), C.byref(n)), what)
    return torch.empty(n.value, dtype=torch.uint8, device=ref.device), n.value


def _lengths(lengths, batch, ref):
    import torch
    if lengths is None:
        return None
    _like("lengths", lengths, ref, (batch,), torch.int32)
    return lengths.contiguous()


# ---------------------------------------------------------------------------
# Root-mean-square norm with the residual's addition
# ---------------------------------------------------------------------------
def _norm_rows(t, width):
    """`t` as [rows, width] with contiguous columns."""
    t = t.reshape(-1, width)
    return t if t.stride(-1) == 1 or t.numel() == 0 else t.contiguous()


def _norm_setup(x, residual, weight, eps, group):
    _on_gpu(x, "x")
    code = _code(x, "x")
    _need(x.dim() >= 1 and x.shape[-1] >= 1, "x has no columns")
    width = x.shape[-1]
    if residual is not None:
        _like("residual", residual, x, x.shape)
    _need(weight.device == x.device and tuple(weight.shape) == (width,),
          f"weight: [{width}] on {x.device}")
    wcode = _code(weight, "weight")
    _need(wcode in (F32, code), f"weight is {weight.dtype}: float32 or x's {x.dtype}")
    x2 = _norm_rows(x, width)
    r2 = None if residual is None else _norm_rows(residual, width)
    cfg = QdsNormConfig(ABI_VERSION, code, wcode, width, x2.shape[0], eps, group)
    return cfg, x2, r2, weight.contiguous()


def residual_norm_forward(x, residual, weight, eps: float = 1e-6):
    """h = x + residual, y = h (mean(h^2) + eps)^(-1/2) weight over the last
    dimension.  Returns y, h (x's type and shape) and rstd (float32, a value per
    row).  `residual` may be None; `weight` is float32 or of x's type."""
    import torch
    cfg, x2, r2, w = _norm_setup(x, residual, weight, eps, 0)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    with _on(x):
        _check(lib().qds_residual_norm(
            C.byref(cfg), x2.data_ptr(), x2.stride(0), _ptr(r2), 0 if r2 is None else r2.stride(0),
            w.data_ptr(), y.data_ptr(), h.data_ptr(), rstd.data_ptr(), _stream(x)),
            "qds_residual_norm")
    return y, h, rstd


def residual_norm_fp8(x, residual, weight, eps: float = 1e-6, group: int = 0):
    """The norm with its output in 8 bits: returns q (float8_e4m3fn, x's shape),
    scale (float32, [..., 1], or [..., width / 128] with `group` = 128) and h.
    q * scale is y; scale is the largest |y| of its columns / 448."""
    import torch
    cfg, x2, r2, w = _norm_setup(x, residual, weight, eps, group)
    _need(group == 0 or (group == 128 and cfg.width % 128 == 0),
          f"group: 0, or 128 where it divides the width ({cfg.width}), not {group}")
    q = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
    h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    scale = torch.empty((*x.shape[:-1], cfg.width // group if group else 1), dtype=torch.float32,
                        device=x.device)
    with _on(x):
        _check(lib().qds_residual_norm_fp8(
            C.byref(cfg), x2.data_ptr(), x2.stride(0), _ptr(r2), 0 if r2 is None else r2.stride(0),
            w.data_ptr(), q.data_ptr(), scale.data_ptr(), h.data_ptr(), _stream(x)),
            "qds_residual_norm_fp8")
    return q, scale, h


def residual_norm_backward(dy, dh, h, rstd, weight):
    """Gradients from those of y and of h (`dh` may be None): returns dx (also
    the residual's gradient) and dweight.  h and rstd are the forward call's."""
    import torch
    cfg, h2, _, w = _norm_setup(h, None, weight, 0.0, 0)
    _like("dy", dy, h, h.shape)
    _like("rstd", rstd, h, h.shape[:-1], torch.float32)
    dy2, dh2 = _norm_rows(dy, cfg.width), None
    if dh is not None:
        _like("dh", dh, h, h.shape)
        dh2 = _norm_rows(dh, cfg.width)
    rstd = rstd.contiguous()
    with _on(h):
        ws, size = _workspace(lib().qds_residual_norm_backward_workspace, cfg, h,
                              "qds_residual_norm_backward_workspace")
        dx = torch.empty(h.shape, dtype=h.dtype, device=h.device)
        dw = torch.empty(weight.shape, dtype=weight.dtype, device=h.device)
        _check(lib().qds_residual_norm_backward(
            C.byref(cfg), dy2.data_ptr(), dy2.stride(0), _ptr(dh2),
            0 if dh2 is None else dh2.stride(0), h2.data_ptr(), h2.stride(0), rstd.data_ptr(),
            w.data_ptr(), dx.data_ptr(), dw.data_ptr(), ws.data_ptr(), size, _stream(h)),
            "qds_residual_norm_backward")
    return dx, dw


# ---------------------------------------------------------------------------
# Attention over a sliding window whose first tokens stay visible
# ---------------------------------------------------------------------------
def _window_setup(q, k, v, window, sinks, scale):
    """Checks q, k, v [batch, rows, heads, dim] (or without rows) and makes the configuration."""
    _on_gpu(q, "q")
    code = _code(q, "q")
    _need(q.dim() in (3, 4) and k.dim() == q.dim(), "q, k, v: [batch, rows, heads, dim]")
    batch, heads, dim = q.shape[0], q.shape[-2], q.shape[-1]
    kv_heads = k.shape[-2]
    _like("k", k, q, (*q.shape[:-2], kv_heads, dim))
    _like("v", v, q, k.shape)
    _need(kv_heads >= 1 and heads % kv_heads == 0,
          f"{heads} query heads are no multiple of {kv_heads} key heads")
    _need(window >= 1 and sinks >= 0, f"window {window} >= 1 and sinks {sinks} >= 0")
    return QdsWindowConfig(ABI_VERSION, code, batch, q.shape[1] if q.dim() == 4 else 0, heads,
                           kv_heads, dim, window, sinks, dim ** -0.5 if scale is None else scale)


def window_attention_forward(q, k, v, window: int, sinks: int = 0, lengths=None, scale=None):
    """Row i of q [batch, rows, heads, dim] attends to rows j <= i of k and v
    [batch, rows, kv_heads, dim] with i - j < window or j < sinks.  Query head h
    reads key head h // (heads / kv_heads).  `lengths` (int32 [batch]): rows of
    each batch element; what is behind them is not read and gets 0.  `scale`
    (> 0) multiplies the scores, dim^(-1/2) if None.

    Nothing is read from behind a length.  Before it, v has to be finite: where
    a row is not, rows that do not see it may become not-a-number as well (their
    weight of 0 times infinity), in the same batch element and head.

    Returns o (q's shape) and lse (float32 [batch, heads, rows])."""
    import torch
    _need(q.dim() == 4, "q, k, v: [batch, rows, heads, dim]")
    cfg = _window_setup(q, k, v, window, sinks, scale)
    lengths = _lengths(lengths, cfg.batch, q)
    q, k, v = _rows(q), _rows(k), _rows(v)
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty((cfg.batch, cfg.heads, cfg.length), dtype=torch.float32, device=q.device)
    with _on(q):
        _check(lib().qds_window_forward(C.byref(cfg), _view(q), _view(k), _view(v), _ptr(lengths),
                                        _view(o), lse.data_ptr(), _stream(q)), "qds_window_forward")
    return o, lse


def window_attention_backward(do, q, k, v, o, lse, window: int, sinks: int = 0, lengths=None,
                              scale=None):
    """Gradients dq, dk, dv from o's, with what the forward call saw and gave."""
    import torch
    _need(q.dim() == 4, "q, k, v: [batch, rows, heads, dim]")
    cfg = _window_setup(q, k, v, window, sinks, scale)
    _like("do", do, q, q.shape)
    _like("o", o, q, q.shape)
    _like("lse", lse, q, (cfg.batch, cfg.heads, cfg.length), torch.float32)
    lengths = _lengths(lengths, cfg.batch, q)
    do, q, k, v, o, lse = _rows(do), _rows(q), _rows(k), _rows(v), _rows(o), lse.contiguous()
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
    with _on(q):
        ws, size = _workspace(lib().qds_window_backward_workspace, cfg, q,
                              "qds_window_backward_workspace")
        _check(lib().qds_window_backward(
            C.byref(cfg), _view(do), _view(q), _view(k), _view(v), _view(o), lse.data_ptr(),
            _ptr(lengths), _view(dq), _view(dk), _view(dv), ws.data_ptr(), size, _stream(q)),
            "qds_window_backward")
    return dq, dk, dv


def window_cache(batch: int, kv_heads: int, dim: int, window: int, sinks: int, dtype, device="cuda:0"):
    """An empty ring cache: k and v, each [batch, kv_heads, sinks + window, dim]."""
    import torch
    shape = (batch, kv_heads, sinks + window, dim)
    return torch.zeros(shape, dtype=dtype, device=device), torch.zeros(shape, dtype=dtype, device=device)


def _cache(cfg, q, k_cache, v_cache):
    shape = (cfg.batch, cfg.kv_heads, cfg.sinks + cfg.window, cfg.dim)
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        _like(name, t, q, shape)
        _need(t.is_contiguous() and t.data_ptr() % 16 == 0, f"{name}: contiguous and 16-byte aligned")


def window_cache_fill(k, v, k_cache, v_cache, window: int, sinks: int = 0, lengths=None):
    """Writes the rows of a prompt (k, v as for window_attention) that later
    tokens can still see into the cache: after it, the token at position
    lengths[b] (or rows) is next."""
    _need(k.dim() == 4, "k, v: [batch, rows, kv_heads, dim]")
    cfg = _window_setup(k, k, v, window, sinks, 1.0)
    _cache(cfg, k, k_cache, v_cache)
    lengths = _lengths(lengths, cfg.batch, k)
    k, v = _rows(k), _rows(v)
    with _on(k):
        _check(lib().qds_window_cache_fill(C.byref(cfg), _view(k), _view(v), _ptr(lengths),
                                           k_cache.data_ptr(), v_cache.data_ptr(), _stream(k)),
               "qds_window_cache_fill")


def window_attention_step(q, k, v, k_cache, v_cache, pos, window: int, sinks: int = 0, scale=None):
    """One token of each batch element: writes k, v [batch, kv_heads, dim] of
    position pos[b] (int32) into the cache and attends with q [batch, heads,
    dim] to what that position sees.  pos[b] < 0: no token; the cache stays and
    the output is 0.  Returns o [batch, heads, dim]."""
    import torch
    _need(q.dim() == 3, "q, k, v: [batch, heads, dim]")
    cfg = _window_setup(q, k, v, window, sinks, scale)
    _cache(cfg, q, k_cache, v_cache)
    _like("pos", pos, q, (cfg.batch,), torch.int32)
    pos = pos.contiguous()
    q, k, v = _rows(q), _rows(k), _rows(v)
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    with _on(q):
        ws, size = _workspace(lib().qds_window_step_workspace, cfg, q, "qds_window_step_workspace")
        _check(lib().qds_window_step(
            C.byref(cfg), _view(q), _view(k), _view(v), k_cache.data_ptr(), v_cache.data_ptr(),
            pos.data_ptr(), _view(o), ws.data_ptr(), size, _stream(q)), "qds_window_step")
    return o


# ---------------------------------------------------------------------------
# Linear attention with a decay for each head
# ---------------------------------------------------------------------------
def _decay_setup(q, k, v, log_decay, scale):
    import torch
    _on_gpu(q, "q")
    code = _code(q, "q")
    _need(q.dim() in (3, 4) and v.dim() == q.dim(), "q, k, v: [batch, rows, heads, dim]")
    _like("k", k, q, q.shape)
    _like("v", v, q, (*q.shape[:-1], v.shape[-1]))
    _like("log_decay", log_decay, q, (q.shape[-2],), torch.float32)
    dim_k, dim_v = q.shape[-1], v.shape[-1]
    return QdsDecayConfig(ABI_VERSION, code, q.shape[0], q.shape[1] if q.dim() == 4 else 0,
                          q.shape[-2], dim_k, dim_v, dim_k ** -0.5 if scale is None else scale)


def _state(name, t, cfg, ref):
    import torch
    if t is None:
        return None
    _like(name, t, ref, (cfg.batch, cfg.heads, cfg.dim_k, cfg.dim_v), torch.float32)
    return t.contiguous()


def decay_attention_forward(q, k, v, log_decay, state=None, lengths=None, scale=None):
    """S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale q_t S_t over the
    rows of q, k [batch, rows, heads, dim_k] and v [batch, rows, heads, dim_v].
    `log_decay` (float32 [heads], <= 0) is a constant of the layer: there is no
    gradient for it.  `state` (float32 [batch, heads, dim_k, dim_v]) is S
    before the first row, 0 if None; `lengths` as for window_attention.

    Returns o and the state after the last row."""
    import torch
    _need(q.dim() == 4, "q, k, v: [batch, rows, heads, dim]")
    cfg = _decay_setup(q, k, v, log_decay, scale)
    state = _state("state", state, cfg, q)
    lengths = _lengths(lengths, cfg.batch, q)
    log_decay = log_decay.contiguous()
    q, k, v = _rows(q), _rows(k), _rows(v)
    o = torch.empty((*q.shape[:-1], cfg.dim_v), dtype=q.dtype, device=q.device)
    last = torch.empty((cfg.batch, cfg.heads, cfg.dim_k, cfg.dim_v), dtype=torch.float32, device=q.device)
    with _on(q):
        ws, size = _workspace(lib().qds_decay_forward_workspace, cfg, q, "qds_decay_forward_workspace")
        _check(lib().qds_decay_forward(
            C.byref(cfg), _view(q), _view(k), _view(v), log_decay.data_ptr(), _ptr(state),
            _ptr(lengths), _view(o), last.data_ptr(), ws.data_ptr(), size, _stream(q)),
            "qds_decay_forward")
    return o, last


def decay_attention_backward(do, q, k, v, log_decay, state=None, dstate=None, lengths=None, scale=None):
    """Gradients dq, dk, dv and that of the first state from those of o and of
    the last state (`dstate`; None: 0)."""
    import torch
    _need(q.dim() == 4, "q, k, v: [batch, rows, heads, dim]")
    cfg = _decay_setup(q, k, v, log_decay, scale)
    _like("do", do, v, v.shape)
    state = _state("state", state, cfg, q)
    dstate = _state("dstate", dstate, cfg, q)
    lengths = _lengths(lengths, cfg.batch, q)
    log_decay = log_decay.contiguous()
    do, q, k, v = _rows(do), _rows(q), _rows(k), _rows(v)
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
    dfirst = torch.empty((cfg.batch, cfg.heads, cfg.dim_k, cfg.dim_v), dtype=torch.float32, device=q.device)
    with _on(q):
        ws, size = _workspace(lib().qds_decay_backward_workspace, cfg, q, "qds_decay_backward_workspace")
        _check(lib().qds_decay_backward(
            C.byref(cfg), _view(do), _view(q), _view(k), _view(v), log_decay.data_ptr(), _ptr(state),
            _ptr(dstate), _ptr(lengths), _view(dq), _view(dk), _view(dv), dfirst.data_ptr(),
            ws.data_ptr(), size, _stream(q)), "qds_decay_backward")
    return dq, dk, dv, dfirst


def decay_attention_step(q, k, v, log_decay, state, scale=None, out_state=None):
    """One token: q, k [batch, heads, dim_k], v [batch, heads, dim_v].  Writes
    the new state into `out_state` (by default into `state` itself) and returns
    o [batch, heads, dim_v] and that state."""
    import torch
    _need(q.dim() == 3, "q, k, v: [batch, heads, dim]")
    cfg = _decay_setup(q, k, v, log_decay, scale)
    out_state = state if out_state is None else out_state
    for name, t in (("state", state), ("out_state", out_state)):
        _like(name, t, q, (cfg.batch, cfg.heads, cfg.dim_k, cfg.dim_v), torch.float32)
        _need(t.is_contiguous() and t.data_ptr() % 16 == 0, f"{name}: contiguous and 16-byte aligned")
    log_decay = log_decay.contiguous()
    q, k, v = _rows(q), _rows(k), _rows(v)
    o = torch.empty((*q.shape[:-1], cfg.dim_v), dtype=q.dtype, device=q.device)
    with _on(q):
        _check(lib().qds_decay_step(C.byref(cfg), _view(q), _view(k), _view(v), log_decay.data_ptr(),
                                    state.data_ptr(), _view(o), out_state.data_ptr(), _stream(q)),
               "qds_decay_step")
    return o, out_state


# ---------------------------------------------------------------------------
# Under autograd
# ---------------------------------------------------------------------------
_functions = None


def _autograd():
    """The autograd functions (torch is imported on first use, as elsewhere in the package)."""
    global _functions
    if _functions is not None:
        return _functions
    import torch

    class ResidualNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, residual, weight, eps):
            y, h, rstd = residual_norm_forward(x, residual, weight, eps)
            ctx.save_for_backward(h, rstd, weight)
            ctx.has_residual = residual is not None
            ctx.set_materialize_grads(False)
            return y, h

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy, dh):
            h, rstd, weight = ctx.saved_tensors
            if dy is None:
                return dh, dh if ctx.has_residual else None, None, None
            dx, dw = residual_norm_backward(dy, dh, h, rstd, weight)
            return dx, dx if ctx.has_residual else None, dw, None

    class WindowAttention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, lengths, window, sinks, scale):
            o, lse = window_attention_forward(q, k, v, window, sinks, lengths, scale)
            ctx.save_for_backward(q, k, v, o, lse, lengths)
            ctx.how = (window, sinks, scale)
            return o

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, do):
            q, k, v, o, lse, lengths = ctx.saved_tensors
            window, sinks, scale = ctx.how
            dq, dk, dv = window_attention_backward(do, q, k, v, o, lse, window, sinks, lengths, scale)
            return dq, dk, dv, None, None, None, None

    class DecayAttention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, log_decay, state, lengths, scale):
            o, last = decay_attention_forward(q, k, v, log_decay, state, lengths, scale)
            ctx.save_for_backward(q, k, v, log_decay, state, lengths)
            ctx.scale = scale
            ctx.set_materialize_grads(False)
            return o, last

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, do, dlast):
            q, k, v, log_decay, state, lengths = ctx.saved_tensors
            if do is None:
                do = torch.zeros_like(v)
            dq, dk, dv, dfirst = decay_attention_backward(do, q, k, v, log_decay, state, dlast, lengths,
                                                          ctx.scale)
            return dq, dk, dv, None, None if state is None else dfirst, None, None

    _functions = (ResidualNorm, WindowAttention, DecayAttention)
    return _functions


def residual_norm(x, residual, weight, eps: float = 1e-6):
    """residual_norm_forward under autograd: returns y and h."""
    return _autograd()[0].apply(x, residual, weight, eps)


def window_attention(q, k, v, window: int, sinks: int = 0, lengths=None, scale=None):
    """window_attention_forward under autograd: returns o."""
    return _autograd()[1].apply(q, k, v, lengths, window, sinks, scale)


def decay_attention(q, k, v, log_decay, state=None, lengths=None, scale=None):
    """decay_attention_forward under autograd: returns o and the last state."""
    _need(not log_decay.requires_grad, "log_decay is a constant of the layer: it has no gradient")
    return _autograd()[2].apply(q, k, v, log_decay, state, lengths, scale)
