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
at multiples of 16 bytes and are less than 2^23 elements apart; others are copied first.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

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
    # stride[0], stride[1], stride[2] of the C struct
    _fields_ = [("data", C.c_void_p), ("stride_b", C.c_int64), ("stride_t", C.c_int64),
                ("stride_h", C.c_int64)]


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
# A rollout calls these operators once per step and layer, so the time of a call
# counts: checks format their messages only when they fail, and what follows from
# shapes, types and devices alone (their checks, the configuration, the size of its
# scratch memory) is worked out once for each set of them.
_CODES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_PLANS = 4096                                      # sets of sizes that are remembered


def _code(t, name):
    code = _CODES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name}: float32, bfloat16 or float16, not {t.dtype}")
    return code


def _like(name, t, ref, shape, dtype=None):
    """Checks a tensor's device, type and shape against those of `ref`."""
    if t.device != ref.device:
        raise ValueError(f"{name} is on {t.device}, not on {ref.device}")
    if t.dtype != (dtype or ref.dtype):
        raise ValueError(f"{name} is {t.dtype}, not {dtype or ref.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} is {tuple(t.shape)}, not {tuple(shape)}")


def _on_gpu(t, name):
    if not t.is_cuda:
        raise RuntimeError(f"{name}: libqdseq needs tensors on a GPU, not on {t.device}")


_FAR = 1 << 23                                     # elements; the kernels take rows that are nearer


def _rows(t):
    """`t` with contiguous, 16-byte aligned rows that are near enough: itself, or a copy."""
    s = t.stride()
    if s[-1] == 1 and t.data_ptr() % 16 == 0 and (len(s) == 3 or -_FAR < s[1] < _FAR or t.shape[1] < 2):
        for x in s[:-1]:
            if x % 8:
                break
        else:
            return t
    return t.clone(memory_format=torch.contiguous_format)


def _view(t):
    """A [batch, rows, heads, dim] or [batch, heads, dim] tensor as a qds_view."""
    s = t.stride()
    return QdsView(t.data_ptr(), s[0], s[1] if len(s) == 4 else 0, s[-2])


def _ptr(t):
    return None if t is None else t.data_ptr()


# The current stream's handle without a Stream object around it, where torch offers that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t):
    if _raw_stream is not None:
        return _raw_stream(t.device.index)
    return torch.cuda.current_stream(t.device).cuda_stream


class _Same:
    """Stands for torch.cuda.device where the tensors' device is the current one."""

    def __enter__(self):
        pass

    def __exit__(self, *exc):
        pass


_same = _Same()


def _on(t):
    index = t.device.index
    return _same if torch.cuda.current_device() == index else torch.cuda.device(index)


_plans = {}


def _remember(key, plan):
    if len(_plans) >= _PLANS:
        _plans.clear()
    _plans[key] = plan
    return plan


def _plan(kind, query, *fields):
    """A configuration, a pointer to it, and the bytes of scratch memory that a call
    with it needs (`query`: the library's function for that, or None)."""
    for x in fields:
        if isinstance(x, int) and not -1 << 31 <= x < 1 << 31:
            raise ValueError(f"{x} is too large")      # ctypes would cut it to 32 bits
    cfg, size = kind(ABI_VERSION, *fields), C.c_uint64(0)
    if query is not None:
        _check(getattr(lib(), query)(C.byref(cfg), C.byref(size)), query)
    return cfg, C.byref(cfg), size.value


def _scratch(size, ref):
    """Scratch memory; torch's allocator keeps it from other work until this
    stream's work on it is done."""
    return ref.new_empty(size, dtype=torch.uint8) if size else None


def _lengths(lengths, batch, ref):
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


def _norm_setup(x, residual, weight, eps, group, query=None):
    key = (x.shape, x.dtype, x.device, weight.shape, weight.dtype, weight.device, eps, group, query) + (
        () if residual is None else (residual.shape, residual.dtype, residual.device))
    plan = _plans.get(key)
    if plan is None:
        _on_gpu(x, "x")
        code = _code(x, "x")
        if x.dim() < 1 or x.shape[-1] < 1:
            raise ValueError("x has no columns")
        width = x.shape[-1]
        if residual is not None:
            _like("residual", residual, x, x.shape)
        if weight.device != x.device or weight.shape != (width,):
            raise ValueError(f"weight: [{width}] on {x.device}")
        wcode = _code(weight, "weight")
        if wcode != F32 and wcode != code:
            raise ValueError(f"weight is {weight.dtype}: float32 or x's {x.dtype}")
        plan = _remember(key, _plan(QdsNormConfig, query, code, wcode, width, x.numel() // width, eps, group))
    width = plan[0].width
    return plan, _norm_rows(x, width), None if residual is None else _norm_rows(residual, width), weight.contiguous()


def residual_norm_forward(x, residual, weight, eps: float = 1e-6):
    """h = x + residual, y = h (mean(h^2) + eps)^(-1/2) weight over the last
    dimension.  Returns y, h (x's type and shape) and rstd (float32, a value per
    row).  `residual` may be None; `weight` is float32 or of x's type."""
    (_, cfg, _), x2, r2, w = _norm_setup(x, residual, weight, eps, 0)
    y, h = x.new_empty(x.shape), x.new_empty(x.shape)
    rstd = x.new_empty(x.shape[:-1], dtype=torch.float32)
    with _on(x):
        _check(lib().qds_residual_norm(
            cfg, x2.data_ptr(), x2.stride(0), _ptr(r2), 0 if r2 is None else r2.stride(0),
            w.data_ptr(), y.data_ptr(), h.data_ptr(), rstd.data_ptr(), _stream(x)),
            "qds_residual_norm")
    return y, h, rstd


def residual_norm_fp8(x, residual, weight, eps: float = 1e-6, group: int = 0):
    """The norm with its output in 8 bits: returns q (float8_e4m3fn, x's shape),
    scale (float32, [..., 1], or [..., width / 128] with `group` = 128) and h.
    q * scale is y; scale is the largest |y| of its columns / 448."""
    (c, cfg, _), x2, r2, w = _norm_setup(x, residual, weight, eps, group)
    if group != 0 and (group != 128 or c.width % 128):
        raise ValueError(f"group: 0, or 128 where it divides the width ({c.width}), not {group}")
    q, h = x.new_empty(x.shape, dtype=torch.float8_e4m3fn), x.new_empty(x.shape)
    scale = x.new_empty((*x.shape[:-1], c.width // group if group else 1), dtype=torch.float32)
    with _on(x):
        _check(lib().qds_residual_norm_fp8(
            cfg, x2.data_ptr(), x2.stride(0), _ptr(r2), 0 if r2 is None else r2.stride(0),
            w.data_ptr(), q.data_ptr(), scale.data_ptr(), h.data_ptr(), _stream(x)),
            "qds_residual_norm_fp8")
    return q, scale, h


def residual_norm_backward(dy, dh, h, rstd, weight):
    """Gradients from those of y and of h (`dh` may be None): returns dx (also
    the residual's gradient) and dweight.  h and rstd are the forward call's."""
    (c, cfg, size), h2, _, w = _norm_setup(h, None, weight, 0.0, 0, "qds_residual_norm_backward_workspace")
    _like("dy", dy, h, h.shape)
    _like("rstd", rstd, h, h.shape[:-1], torch.float32)
    dy2, dh2 = _norm_rows(dy, c.width), None
    if dh is not None:
        _like("dh", dh, h, h.shape)
        dh2 = _norm_rows(dh, c.width)
    rstd = rstd.contiguous()
    with _on(h):
        ws = _scratch(size, h)
        dx, dw = h.new_empty(h.shape), weight.new_empty(weight.shape)
        _check(lib().qds_residual_norm_backward(
            cfg, dy2.data_ptr(), dy2.stride(0), _ptr(dh2),
            0 if dh2 is None else dh2.stride(0), h2.data_ptr(), h2.stride(0), rstd.data_ptr(),
            w.data_ptr(), dx.data_ptr(), dw.data_ptr(), _ptr(ws), size, _stream(h)),
            "qds_residual_norm_backward")
    return dx, dw


# ---------------------------------------------------------------------------
# Attention over a sliding window whose first tokens stay visible
# ---------------------------------------------------------------------------
def _window_setup(q, k, v, window, sinks, scale, rows, query=None):
    """Checks q, k, v [batch, rows, heads, dim] (or without rows) and makes the plan."""
    key = (q.shape, q.dtype, q.device, k.shape, k.dtype, k.device, v.shape, v.dtype, v.device, window, sinks,
           scale, rows, query)
    plan = _plans.get(key)
    if plan is not None:
        return plan
    _on_gpu(q, "q")
    code = _code(q, "q")
    if q.dim() != (4 if rows else 3) or k.dim() != q.dim():
        raise ValueError("q, k, v: [batch, rows, heads, dim]" if rows else "q, k, v: [batch, heads, dim]")
    batch, heads, dim = q.shape[0], q.shape[-2], q.shape[-1]
    kv_heads = k.shape[-2]
    _like("k", k, q, (*q.shape[:-2], kv_heads, dim))
    _like("v", v, q, k.shape)
    if kv_heads < 1 or heads % kv_heads:
        raise ValueError(f"{heads} query heads are no multiple of {kv_heads} key heads")
    if window < 1 or sinks < 0:
        raise ValueError(f"window {window} >= 1 and sinks {sinks} >= 0")
    return _remember(key, _plan(QdsWindowConfig, query, code, batch, q.shape[1] if rows else 0, heads, kv_heads,
                                dim, window, sinks, dim ** -0.5 if scale is None else scale))


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
    c, cfg, _ = _window_setup(q, k, v, window, sinks, scale, True)
    lengths = _lengths(lengths, c.batch, q)
    q, k, v = _rows(q), _rows(k), _rows(v)
    o = q.new_empty(q.shape)
    lse = q.new_empty((c.batch, c.heads, c.length), dtype=torch.float32)
    with _on(q):
        _check(lib().qds_window_forward(cfg, _view(q), _view(k), _view(v), _ptr(lengths),
                                        _view(o), lse.data_ptr(), _stream(q)), "qds_window_forward")
    return o, lse


def window_attention_backward(do, q, k, v, o, lse, window: int, sinks: int = 0, lengths=None,
                              scale=None):
    """Gradients dq, dk, dv from o's, with what the forward call saw and gave."""
    c, cfg, size = _window_setup(q, k, v, window, sinks, scale, True, "qds_window_backward_workspace")
    _like("do", do, q, q.shape)
    _like("o", o, q, q.shape)
    _like("lse", lse, q, (c.batch, c.heads, c.length), torch.float32)
    lengths = _lengths(lengths, c.batch, q)
    do, q, k, v, o, lse = _rows(do), _rows(q), _rows(k), _rows(v), _rows(o), lse.contiguous()
    dq, dk, dv = q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape)
    with _on(q):
        ws = _scratch(size, q)
        _check(lib().qds_window_backward(
            cfg, _view(do), _view(q), _view(k), _view(v), _view(o), lse.data_ptr(),
            _ptr(lengths), _view(dq), _view(dk), _view(dv), _ptr(ws), size, _stream(q)),
            "qds_window_backward")
    return dq, dk, dv


def window_cache(batch: int, kv_heads: int, dim: int, window: int, sinks: int, dtype, device="cuda:0"):
    """An empty ring cache: k and v, each [batch, kv_heads, sinks + window, dim]."""
    shape = (batch, kv_heads, sinks + window, dim)
    return torch.zeros(shape, dtype=dtype, device=device), torch.zeros(shape, dtype=dtype, device=device)


def _in_place(name, t, ref, shape, dtype=None):
    _like(name, t, ref, shape, dtype)
    if not t.is_contiguous() or t.data_ptr() % 16:
        raise ValueError(f"{name}: contiguous and 16-byte aligned")


def _cache(c, q, k_cache, v_cache):
    shape = (c.batch, c.kv_heads, c.sinks + c.window, c.dim)
    _in_place("k_cache", k_cache, q, shape)
    _in_place("v_cache", v_cache, q, shape)


def window_cache_fill(k, v, k_cache, v_cache, window: int, sinks: int = 0, lengths=None):
    """Writes the rows of a prompt (k, v as for window_attention) that later
    tokens can still see into the cache: after it, the token at position
    lengths[b] (or rows) is next."""
    c, cfg, _ = _window_setup(k, k, v, window, sinks, 1.0, True)
    _cache(c, k, k_cache, v_cache)
    lengths = _lengths(lengths, c.batch, k)
    k, v = _rows(k), _rows(v)
    with _on(k):
        _check(lib().qds_window_cache_fill(cfg, _view(k), _view(v), _ptr(lengths),
                                           k_cache.data_ptr(), v_cache.data_ptr(), _stream(k)),
               "qds_window_cache_fill")


def window_attention_step(q, k, v, k_cache, v_cache, pos, window: int, sinks: int = 0, scale=None):
    """One token of each batch element: writes k, v [batch, kv_heads, dim] of
    position pos[b] (int32) into the cache and attends with q [batch, heads,
    dim] to what that position sees.  pos[b] < 0: no token; the cache stays and
    the output is 0.  Returns o [batch, heads, dim]."""
    c, cfg, size = _window_setup(q, k, v, window, sinks, scale, False, "qds_window_step_workspace")
    _cache(c, q, k_cache, v_cache)
    _like("pos", pos, q, (c.batch,), torch.int32)
    pos = pos.contiguous()
    q, k, v = _rows(q), _rows(k), _rows(v)
    o = q.new_empty(q.shape)
    with _on(q):
        ws = _scratch(size, q)
        _check(lib().qds_window_step(
            cfg, _view(q), _view(k), _view(v), k_cache.data_ptr(), v_cache.data_ptr(),
            pos.data_ptr(), _view(o), _ptr(ws), size, _stream(q)), "qds_window_step")
    return o


# ---------------------------------------------------------------------------
# Linear attention with a decay for each head
# ---------------------------------------------------------------------------
def _decay_setup(q, k, v, log_decay, scale, rows, query=None):
    key = (q.shape, q.dtype, q.device, k.shape, k.dtype, k.device, v.shape, v.dtype, v.device, log_decay.shape,
           log_decay.dtype, log_decay.device, scale, rows, query)
    plan = _plans.get(key)
    if plan is not None:
        return plan
    _on_gpu(q, "q")
    code = _code(q, "q")
    if q.dim() != (4 if rows else 3) or v.dim() != q.dim():
        raise ValueError("q, k, v: [batch, rows, heads, dim]" if rows else "q, k, v: [batch, heads, dim]")
    heads, dim_k, dim_v = q.shape[-2], q.shape[-1], v.shape[-1]
    _like("k", k, q, q.shape)
    _like("v", v, q, (*q.shape[:-1], dim_v))
    _like("log_decay", log_decay, q, (heads,), torch.float32)
    return _remember(key, _plan(QdsDecayConfig, query, code, q.shape[0], q.shape[1] if rows else 0, heads, dim_k,
                                dim_v, dim_k ** -0.5 if scale is None else scale))


def _state(name, t, c, ref):
    if t is None:
        return None
    _like(name, t, ref, (c.batch, c.heads, c.dim_k, c.dim_v), torch.float32)
    return t.contiguous()


def decay_attention_forward(q, k, v, log_decay, state=None, lengths=None, scale=None):
    """S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale q_t S_t over the
    rows of q, k [batch, rows, heads, dim_k] and v [batch, rows, heads, dim_v].
    `log_decay` (float32 [heads], <= 0) is a constant of the layer: there is no
    gradient for it.  `state` (float32 [batch, heads, dim_k, dim_v]) is S
    before the first row, 0 if None; `lengths` as for window_attention.

    Nothing is read from behind a length.  Before it, k and v have to be finite:
    a row that is not may make up to 63 rows before it not-a-number as well
    (their weight of 0 times infinity), in the same batch element and head.
    States may hold any float32 numbers, in float16, too.

    Returns o and the state after the last row."""
    cfg, ref, size = _decay_setup(q, k, v, log_decay, scale, True, "qds_decay_forward_workspace")
    state = _state("state", state, cfg, q)
    lengths = _lengths(lengths, cfg.batch, q)
    log_decay = log_decay.contiguous()
    q, k, v = _rows(q), _rows(k), _rows(v)
    o = v.new_empty(v.shape)
    last = q.new_empty((cfg.batch, cfg.heads, cfg.dim_k, cfg.dim_v), dtype=torch.float32)
    with _on(q):
        ws = _scratch(size, q)
        _check(lib().qds_decay_forward(
            ref, _view(q), _view(k), _view(v), log_decay.data_ptr(), _ptr(state),
            _ptr(lengths), _view(o), last.data_ptr(), _ptr(ws), size, _stream(q)),
            "qds_decay_forward")
    return o, last


def decay_attention_backward(do, q, k, v, log_decay, state=None, dstate=None, lengths=None, scale=None):
    """Gradients dq, dk, dv and that of the first state from those of o and of
    the last state (`dstate`; None: 0)."""
    cfg, ref, size = _decay_setup(q, k, v, log_decay, scale, True, "qds_decay_backward_workspace")
    _like("do", do, v, v.shape)
    state = _state("state", state, cfg, q)
    dstate = _state("dstate", dstate, cfg, q)
    lengths = _lengths(lengths, cfg.batch, q)
    log_decay = log_decay.contiguous()
    do, q, k, v = _rows(do), _rows(q), _rows(k), _rows(v)
    dq, dk, dv = q.new_empty(q.shape), k.new_empty(k.shape), v.new_empty(v.shape)
    dfirst = q.new_empty((cfg.batch, cfg.heads, cfg.dim_k, cfg.dim_v), dtype=torch.float32)
    with _on(q):
        ws = _scratch(size, q)
        _check(lib().qds_decay_backward(
            ref, _view(do), _view(q), _view(k), _view(v), log_decay.data_ptr(), _ptr(state),
            _ptr(dstate), _ptr(lengths), _view(dq), _view(dk), _view(dv), dfirst.data_ptr(),
            _ptr(ws), size, _stream(q)), "qds_decay_backward")
    return dq, dk, dv, dfirst


def decay_attention_step(q, k, v, log_decay, state, scale=None, out_state=None):
    """One token: q, k [batch, heads, dim_k], v [batch, heads, dim_v].  Writes
    the new state into `out_state` (by default into `state` itself) and returns
    o [batch, heads, dim_v] and that state."""
    cfg, ref, _ = _decay_setup(q, k, v, log_decay, scale, False)
    out_state = state if out_state is None else out_state
    shape = (cfg.batch, cfg.heads, cfg.dim_k, cfg.dim_v)
    _in_place("state", state, q, shape, torch.float32)
    if out_state is not state:
        _in_place("out_state", out_state, q, shape, torch.float32)
    log_decay = log_decay.contiguous()
    q, k, v = _rows(q), _rows(k), _rows(v)
    o = v.new_empty(v.shape)
    with _on(q):
        _check(lib().qds_decay_step(ref, _view(q), _view(k), _view(v), log_decay.data_ptr(),
                                    state.data_ptr(), _view(o), out_state.data_ptr(), _stream(q)),
               "qds_decay_step")
    return o, out_state


# ---------------------------------------------------------------------------
# Under autograd
# ---------------------------------------------------------------------------
_functions = None


def _autograd():
    """The autograd functions, made on first use."""
    global _functions
    if _functions is not None:
        return _functions

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
    if log_decay.requires_grad:
        raise ValueError("log_decay is a constant of the layer: it has no gradient")
    return _autograd()[2].apply(q, k, v, log_decay, state, lengths, scale)
