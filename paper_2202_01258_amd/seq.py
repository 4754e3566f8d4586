"""Operators of sequence policies over episodes: Python binding of libqdseq.so
(the C ABI of include/qd_seq.h).

A sequence policy is told the wanted descriptor in its first tokens and reads
one token per step of an episode; it is fitted to the episodes of an archive's
elites, or rolled out in their place.  Its blocks are made of

  residual_norm        root-mean-square norm with the residual's addition
  window_attention     attention over a sliding window whose first tokens stay visible
  decay_attention      linear attention with a decay for each head
  causal_conv          a short convolution over the rows, for each column
  selective_scan       a state space scan whose steps and inputs the tokens choose
  branch_norm          the norms after and before a block with its gate and the residual's scale
  dropout              from a counter: its mask is never stored

Each is differentiable under torch's autograd.  The calls below them are the
plain ones: `*_forward` and `*_backward` for programs that keep their own
tape, `residual_norm_fp8` for an 8-bit output, and `window_attention_step`
(with `window_cache` and `window_cache_fill`), `decay_attention_step`,
`causal_conv_step` and `selective_scan_step` for rollouts, one token at a time.

Argument marshalling only: outputs and scratch memory are torch tensors, work
is enqueued on torch's current stream of the tensors' device, nothing waits for
the GPU, and there is no fallback.  Tensors are used on that stream alone; a
tensor made on another stream has to be synchronised with it first, as for any
torch operation.  As for any autograd function, too, a backward pass is captured
into a graph only while no eager graph of the same leaves lives: torch would wait
for that one's stream within the capture.

Attention takes bfloat16 or float16 tensors whose rows start at multiples of 16
bytes and are less than 2^23 elements apart; others are copied first.  The other
operators take float32, too, and rows of any alignment; they copy tensors whose
columns are apart (the scan those with rows 2^23 elements apart or more, dropout
those that are not contiguous).
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
           "qds_causal_conv", "qds_causal_conv_backward_workspace", "qds_causal_conv_backward",
           "qds_causal_conv_step", "qds_selective_scan_marks", "qds_selective_scan_workspace",
           "qds_selective_scan", "qds_selective_scan_backward_workspace",
           "qds_selective_scan_backward", "qds_selective_scan_step", "qds_branch_norm",
           "qds_branch_norm_backward_workspace", "qds_branch_norm_backward", "qds_dropout",
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


class QdsRows(C.Structure):
    # stride[0], stride[1] of the C struct
    _fields_ = [("data", C.c_void_p), ("stride_b", C.c_int64), ("stride_t", C.c_int64)]


class QdsConvConfig(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("dtype", C.c_int32), ("weight_dtype", C.c_int32),
                ("batch", C.c_int32), ("length", C.c_int32), ("width", C.c_int32),
                ("taps", C.c_int32), ("silu", C.c_int32)]


class QdsScanConfig(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("dtype", C.c_int32), ("batch", C.c_int32),
                ("length", C.c_int32), ("width", C.c_int32), ("states", C.c_int32)]


class QdsBranchConfig(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("dtype", C.c_int32), ("weight_dtype", C.c_int32),
                ("width", C.c_int32), ("rows", C.c_int64), ("eps", C.c_float),
                ("residual_scale", C.c_float)]


class QdsDropoutConfig(C.Structure):
    _fields_ = [("abi_version", C.c_uint32), ("dtype", C.c_int32), ("elements", C.c_int64),
                ("threshold", C.c_uint32), ("site", C.c_uint32)]


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
        R, K, S = QdsRows, C.POINTER(QdsConvConfig), C.POINTER(QdsScanConfig)
        L.qds_causal_conv.argtypes = [K, R, P, P, P, P, R, P, P]
        L.qds_causal_conv_backward_workspace.argtypes = [K, B]
        L.qds_causal_conv_backward.argtypes = [K, R, R, P, P, P, P, P, R, P, P, P, P, U, P]
        L.qds_causal_conv_step.argtypes = [K, R, P, P, P, R, P, P]
        L.qds_selective_scan_marks.argtypes = [S, B]
        L.qds_selective_scan_workspace.argtypes = [S, B]
        L.qds_selective_scan.argtypes = [S, R, R, P, R, R, P, R, P, P, P, P, P, P, P, U, P]
        L.qds_selective_scan_backward_workspace.argtypes = [S, B]
        L.qds_selective_scan_backward.argtypes = [S, R, R, R, P, R, R, P, R, P, P, P, P, P, P, P, P, P, P, P, P,
                                                  P, P, U, P]
        L.qds_selective_scan_step.argtypes = [S, R, R, P, R, R, P, R, P, P, P, P, P]
        L.qds_branch_norm.argtypes = [C.POINTER(QdsBranchConfig), P, I, P, I, P, I, P, P, P, P, P, P]
        L.qds_branch_norm_backward_workspace.argtypes = [C.POINTER(QdsBranchConfig), B]
        L.qds_branch_norm_backward.argtypes = [C.POINTER(QdsBranchConfig), P, I, P, I, P, I, P, I, P, I, P, P, P,
                                               P, P, P, P, P, P, U, P]
        L.qds_dropout.argtypes = [C.POINTER(QdsDropoutConfig), P, P, P, P, P]
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
# Short causal convolution
# ---------------------------------------------------------------------------
def _columns(t):
    """`t` with contiguous columns: itself, or a copy."""
    return t if t.stride(-1) == 1 or t.shape[-1] == 1 else t.contiguous()


def _near(t):
    """`t` with contiguous columns and rows that are near enough for the scan: itself, or a copy."""
    t = _columns(t)
    return t if t.dim() < 3 or t.stride(1) < _FAR or t.shape[1] < 2 else t.clone(memory_format=torch.contiguous_format)


_NO_ROWS = QdsRows(None, 0, 0)


def _row_view(t):
    """A [batch, rows, width] or [batch, width] tensor as qds_rows."""
    if t is None:
        return _NO_ROWS
    s = t.stride()
    return QdsRows(t.data_ptr(), s[0], s[1] if len(s) == 3 else 0)


def _sig(t):
    return None if t is None else (t.shape, t.dtype, t.device)


def _written(name, t, ref, shape, dtype):
    """A state that a step writes."""
    _like(name, t, ref, shape, dtype)
    if not t.is_contiguous():
        raise ValueError(f"{name}: contiguous")


def _conv_setup(x, weight, bias, silu, rows, query=None):
    """Checks x [batch, rows, width] (or without rows), weight and bias, and makes the plan."""
    key = ("conv", x.shape, x.dtype, x.device, _sig(weight), _sig(bias), silu, rows, query)
    plan = _plans.get(key)
    if plan is not None:
        return plan
    _on_gpu(x, "x")
    code = _code(x, "x")
    if x.dim() != (3 if rows else 2) or x.shape[-1] < 1:
        raise ValueError("x: [batch, rows, width]" if rows else "x: [batch, width]")
    width = x.shape[-1]
    wcode = _code(weight, "weight")
    if wcode != F32 and wcode != code:
        raise ValueError(f"weight is {weight.dtype}: float32 or x's {x.dtype}")
    if weight.device != x.device or weight.dim() != 2 or weight.shape[1] != width or not 1 <= weight.shape[0] <= 8:
        raise ValueError(f"weight: [taps, {width}] on {x.device}, of 1 to 8 taps")
    if bias is not None:
        _like("bias", bias, weight, (width,))
    return _remember(key, _plan(QdsConvConfig, query, code, wcode, x.shape[0], x.shape[1] if rows else 0, width,
                                weight.shape[0], int(bool(silu))))


def _conv_state(name, t, c, ref):
    if t is None:
        return None
    _like(name, t, ref, (c.batch, c.taps - 1, c.width))
    return t.contiguous()


def causal_conv_forward(x, weight, bias=None, state=None, lengths=None, silu: bool = True):
    """p_t = bias + sum_k weight[k] x_{t - taps + 1 + k} for each column of x [batch, rows,
    width]; y = p sigmoid(p), or p without `silu`.  `weight` [taps, width] (1 to 8 taps) and
    `bias` [width] are float32 or of x's type.  `state` [batch, taps - 1, width] (x's type)
    holds the rows before the first, the oldest first; None: 0.  `lengths` (int32 [batch]):
    rows of each batch element; what is behind them is not read and gets 0.

    Returns y and the state behind the last row."""
    c, cfg, _ = _conv_setup(x, weight, bias, silu, True)
    state = _conv_state("state", state, c, x)
    lengths = _lengths(lengths, c.batch, x)
    x, weight, bias = _columns(x), weight.contiguous(), None if bias is None else bias.contiguous()
    y, last = x.new_empty(x.shape), x.new_empty((c.batch, c.taps - 1, c.width))
    with _on(x):
        _check(lib().qds_causal_conv(cfg, _row_view(x), weight.data_ptr(), _ptr(bias), _ptr(state), _ptr(lengths),
                                     _row_view(y), last.data_ptr(), _stream(x)), "qds_causal_conv")
    return y, last


def causal_conv_backward(dy, x, weight, bias=None, state=None, dlast=None, lengths=None, silu: bool = True):
    """Gradients from those of y and of the last state (`dlast`; None: 0): returns dx, dweight,
    dbias (None without a bias) and that of the first state (also where `state` is None)."""
    c, cfg, size = _conv_setup(x, weight, bias, silu, True, "qds_causal_conv_backward_workspace")
    _like("dy", dy, x, x.shape)
    state, dlast = _conv_state("state", state, c, x), _conv_state("dlast", dlast, c, x)
    lengths = _lengths(lengths, c.batch, x)
    dy, x, weight = _columns(dy), _columns(x), weight.contiguous()
    bias = None if bias is None else bias.contiguous()
    dx, dfirst = x.new_empty(x.shape), x.new_empty((c.batch, c.taps - 1, c.width))
    dw, db = weight.new_empty(weight.shape), None if bias is None else bias.new_empty(bias.shape)
    with _on(x):
        ws = _scratch(size, x)
        _check(lib().qds_causal_conv_backward(
            cfg, _row_view(dy), _row_view(x), weight.data_ptr(), _ptr(bias), _ptr(state), _ptr(dlast), _ptr(lengths),
            _row_view(dx), dw.data_ptr(), _ptr(db), dfirst.data_ptr(), _ptr(ws), size, _stream(x)),
            "qds_causal_conv_backward")
    return dx, dw, db, dfirst


def causal_conv_step(x, weight, bias, state, silu: bool = True, out_state=None):
    """One row x [batch, width] of each batch element.  Writes the new state into `out_state`
    (by default into `state` itself) and returns y [batch, width] and that state."""
    c, cfg, _ = _conv_setup(x, weight, bias, silu, False)
    out_state = state if out_state is None else out_state
    shape = (c.batch, c.taps - 1, c.width)
    _written("state", state, x, shape, x.dtype)
    if out_state is not state:
        _written("out_state", out_state, x, shape, x.dtype)
    x, weight, bias = _columns(x), weight.contiguous(), None if bias is None else bias.contiguous()
    y = x.new_empty(x.shape)
    with _on(x):
        _check(lib().qds_causal_conv_step(cfg, _row_view(x), weight.data_ptr(), _ptr(bias), state.data_ptr(),
                                          _row_view(y), out_state.data_ptr(), _stream(x)), "qds_causal_conv_step")
    return y, out_state


# ---------------------------------------------------------------------------
# Selective state space scan
# ---------------------------------------------------------------------------
def _scan_setup(u, delta, a, b, c, skip, gate, bias, rows, query=None):
    key = ("scan", u.shape, u.dtype, u.device, _sig(delta), _sig(a), _sig(b), _sig(c), _sig(skip), _sig(gate),
           _sig(bias), rows, query)
    plan = _plans.get(key)
    if plan is not None:
        return plan
    _on_gpu(u, "u")
    code = _code(u, "u")
    if u.dim() != (3 if rows else 2) or u.shape[-1] < 1:
        raise ValueError("u: [batch, rows, width]" if rows else "u: [batch, width]")
    width = u.shape[-1]
    if a.dim() != 2 or not 1 <= a.shape[1] <= 32:
        raise ValueError(f"a: [{width}, states], of 1 to 32 states")
    _like("a", a, u, (width, a.shape[1]), torch.float32)
    _like("delta", delta, u, u.shape)
    _like("b", b, u, (*u.shape[:-1], a.shape[1]))
    _like("c", c, u, b.shape)
    if gate is not None:
        _like("gate", gate, u, u.shape)
    for name, t in (("skip", skip), ("bias", bias)):
        if t is not None:
            _like(name, t, u, (width,), torch.float32)
    fields = code, u.shape[0], u.shape[1] if rows else 0, width, a.shape[1]
    marks = _plan(QdsScanConfig, "qds_selective_scan_marks", *fields)[2] if rows else 0
    return _remember(key, (*_plan(QdsScanConfig, query, *fields), marks))


def _scan_state(name, t, cfg, ref):
    if t is None:
        return None
    _like(name, t, ref, (cfg.batch, cfg.width, cfg.states), torch.float32)
    return t.contiguous()


def _dense(t):
    return None if t is None else t.contiguous()


def selective_scan_forward(u, delta, a, b, c, skip=None, gate=None, bias=None, state=None, lengths=None,
                           keep: bool = False):
    """dt = log(1 + e^(delta + bias)), h_t[n] = e^(dt a[n]) h_{t-1}[n] + dt u_t b_t[n],
    y_t = sum_n c_t[n] h_t[n] + skip u_t for each column of u and delta [batch, rows, width],
    with b and c [batch, rows, states] (1 to 32 states) for all columns; o = y gate
    sigmoid(gate), or y without a gate (u's shape).  `a` [width, states], `skip` and `bias`
    [width] are float32, and so is `state` [batch, width, states], h before the first row (None:
    0).  `lengths` as for causal_conv_forward.  All arithmetic is float32.

    Rows that are not finite reach the rows behind them (those of b and c in every column), as
    in the definition.  batch times width, each row of columns rounded up to a multiple of 64, is
    below 2^30.

    Returns o, the state behind the last row, and with `keep` what selective_scan_backward
    needs of this pass (else None)."""
    cfg, ref, size, room = _scan_setup(u, delta, a, b, c, skip, gate, bias, True, "qds_selective_scan_workspace")
    state = _scan_state("state", state, cfg, u)
    lengths = _lengths(lengths, cfg.batch, u)
    u, delta, b, c = _near(u), _near(delta), _near(b), _near(c)
    a, skip, bias, gate = a.contiguous(), _dense(skip), _dense(bias), None if gate is None else _near(gate)
    o = u.new_empty(u.shape)
    last = u.new_empty((cfg.batch, cfg.width, cfg.states), dtype=torch.float32)
    with _on(u):
        ws = _scratch(size, u)
        marks = u.new_empty(room, dtype=torch.uint8) if keep else None
        _check(lib().qds_selective_scan(
            ref, _row_view(u), _row_view(delta), a.data_ptr(), _row_view(b), _row_view(c), _ptr(skip), _row_view(gate),
            _ptr(bias), _ptr(state), _ptr(lengths), o.data_ptr(), last.data_ptr(), _ptr(marks), _ptr(ws), size,
            _stream(u)), "qds_selective_scan")
    return o, last, marks


def selective_scan_backward(do, u, delta, a, b, c, marks, skip=None, gate=None, bias=None, dlast=None, lengths=None):
    """Gradients from those of o and of the last state (`dlast`; None: 0), with what the forward
    call saw and kept: returns du, ddelta, da, db, dc, dskip, dgate, dbias (None for those that
    are) and that of the first state.  batch times rows is at most 2^25."""
    cfg, ref, size, room = _scan_setup(u, delta, a, b, c, skip, gate, bias, True, "qds_selective_scan_backward_workspace")
    _like("do", do, u, u.shape)
    _like("marks", marks, u, (room,), torch.uint8)
    dlast = _scan_state("dlast", dlast, cfg, u)
    lengths = _lengths(lengths, cfg.batch, u)
    do, u, delta, b, c = _near(do), _near(u), _near(delta), _near(b), _near(c)
    a, skip, bias, gate = a.contiguous(), _dense(skip), _dense(bias), None if gate is None else _near(gate)
    du, ddelta, da = u.new_empty(u.shape), u.new_empty(u.shape), a.new_empty(a.shape)
    db, dc = b.new_empty(b.shape), c.new_empty(c.shape)
    dgate = None if gate is None else u.new_empty(u.shape)
    dskip, dbias = (None if t is None else t.new_empty(t.shape) for t in (skip, bias))
    dfirst = a.new_empty((cfg.batch, cfg.width, cfg.states))
    with _on(u):
        ws = _scratch(size, u)
        _check(lib().qds_selective_scan_backward(
            ref, _row_view(do), _row_view(u), _row_view(delta), a.data_ptr(), _row_view(b), _row_view(c), _ptr(skip),
            _row_view(gate), _ptr(bias), marks.data_ptr(), _ptr(dlast), _ptr(lengths), du.data_ptr(),
            ddelta.data_ptr(), da.data_ptr(), db.data_ptr(), dc.data_ptr(), _ptr(dskip), _ptr(dgate), _ptr(dbias),
            dfirst.data_ptr(), _ptr(ws), size, _stream(u)), "qds_selective_scan_backward")
    return du, ddelta, da, db, dc, dskip, dgate, dbias, dfirst


def selective_scan_step(u, delta, a, b, c, state, skip=None, gate=None, bias=None, out_state=None):
    """One row of each batch element: u, delta, gate [batch, width], b, c [batch, states].
    Writes the new state into `out_state` (by default into `state` itself) and returns
    o [batch, width] and that state."""
    cfg, ref, _, _ = _scan_setup(u, delta, a, b, c, skip, gate, bias, False)
    out_state = state if out_state is None else out_state
    shape = (cfg.batch, cfg.width, cfg.states)
    _written("state", state, u, shape, torch.float32)
    if out_state is not state:
        _written("out_state", out_state, u, shape, torch.float32)
    u, delta, b, c = _columns(u), _columns(delta), _columns(b), _columns(c)
    a, skip, bias, gate = a.contiguous(), _dense(skip), _dense(bias), None if gate is None else _columns(gate)
    o = u.new_empty(u.shape)
    with _on(u):
        _check(lib().qds_selective_scan_step(
            ref, _row_view(u), _row_view(delta), a.data_ptr(), _row_view(b), _row_view(c), _ptr(skip), _row_view(gate),
            _ptr(bias), state.data_ptr(), o.data_ptr(), out_state.data_ptr(), _stream(u)), "qds_selective_scan_step")
    return o, out_state


# ---------------------------------------------------------------------------
# Norms after and before a block, its gate, the residual's scale
# ---------------------------------------------------------------------------
def _branch_setup(x, gate, residual, branch_weight, weight, residual_scale, eps, query=None):
    key = ("branch", x.shape, x.dtype, x.device, _sig(gate), _sig(residual), _sig(branch_weight), _sig(weight),
           residual_scale, eps, query)
    plan = _plans.get(key)
    if plan is not None:
        return plan
    _on_gpu(x, "x")
    code = _code(x, "x")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x has no columns")
    width = x.shape[-1]
    _like("residual", residual, x, x.shape)
    if gate is not None:
        _like("gate", gate, x, x.shape)
    if weight.device != x.device or weight.shape != (width,):
        raise ValueError(f"weight: [{width}] on {x.device}")
    wcode = _code(weight, "weight")
    if wcode != F32 and wcode != code:
        raise ValueError(f"weight is {weight.dtype}: float32 or x's {x.dtype}")
    _like("branch_weight", branch_weight, weight, (width,))
    return _remember(key, _plan(QdsBranchConfig, query, code, wcode, width, x.numel() // width, eps, residual_scale))


def branch_norm_forward(x, gate, residual, branch_weight, weight, residual_scale: float = 1.0, eps: float = 1e-6):
    """The end of a block and the norm in front of the next, over the last dimension:
    n = x (mean(x^2) + eps)^(-1/2) branch_weight, h = residual_scale residual + gate sigmoid(gate) n
    (`gate` None: + n), y = h (mean(h^2) + eps)^(-1/2) weight.  x, gate and residual have one
    shape and type; both weights are float32 or of x's type.

    Returns y, h (x's type and shape) and the factors of both norms (float32 [2, ...])."""
    _, cfg, _ = _branch_setup(x, gate, residual, branch_weight, weight, residual_scale, eps)
    width = x.shape[-1]
    x2, r2, g2 = _norm_rows(x, width), _norm_rows(residual, width), None if gate is None else _norm_rows(gate, width)
    w1, w2 = branch_weight.contiguous(), weight.contiguous()
    y, h = x.new_empty(x.shape), x.new_empty(x.shape)
    rstds = x.new_empty((2, *x.shape[:-1]), dtype=torch.float32)
    with _on(x):
        _check(lib().qds_branch_norm(
            cfg, x2.data_ptr(), x2.stride(0), _ptr(g2), 0 if g2 is None else g2.stride(0), r2.data_ptr(), r2.stride(0),
            w1.data_ptr(), w2.data_ptr(), y.data_ptr(), h.data_ptr(), rstds.data_ptr(), _stream(x)), "qds_branch_norm")
    return y, h, rstds


def branch_norm_backward(dy, dh, x, gate, residual, rstds, branch_weight, weight, residual_scale: float = 1.0):
    """Gradients from those of y and of h (`dh` may be None), with what the forward call saw and
    gave: returns dx, dgate (None without a gate), dresidual, dbranch_weight and dweight."""
    c, cfg, size = _branch_setup(x, gate, residual, branch_weight, weight, residual_scale, 0.0,
                                 "qds_branch_norm_backward_workspace")
    _like("dy", dy, x, x.shape)
    _like("rstds", rstds, x, (2, *x.shape[:-1]), torch.float32)
    x2, r2, dy2 = _norm_rows(x, c.width), _norm_rows(residual, c.width), _norm_rows(dy, c.width)
    g2 = dh2 = None
    if gate is not None:
        g2 = _norm_rows(gate, c.width)
    if dh is not None:
        _like("dh", dh, x, x.shape)
        dh2 = _norm_rows(dh, c.width)
    rstds, w1, w2 = rstds.contiguous(), branch_weight.contiguous(), weight.contiguous()
    dx, dr, dg = x.new_empty(x.shape), x.new_empty(x.shape), None if gate is None else x.new_empty(x.shape)
    dw1, dw2 = weight.new_empty(weight.shape), weight.new_empty(weight.shape)
    with _on(x):
        ws = _scratch(size, x)
        _check(lib().qds_branch_norm_backward(
            cfg, dy2.data_ptr(), dy2.stride(0), _ptr(dh2), 0 if dh2 is None else dh2.stride(0), x2.data_ptr(),
            x2.stride(0), _ptr(g2), 0 if g2 is None else g2.stride(0), r2.data_ptr(), r2.stride(0), rstds.data_ptr(),
            w1.data_ptr(), w2.data_ptr(), dx.data_ptr(), _ptr(dg), dr.data_ptr(), dw1.data_ptr(), dw2.data_ptr(),
            _ptr(ws), size, _stream(x)), "qds_branch_norm_backward")
    return dx, dg, dr, dw1, dw2


# ---------------------------------------------------------------------------
# Dropout from a counter
# ---------------------------------------------------------------------------
def dropout_rng(seed: int, step: int = 0, device="cuda:0"):
    """The state of a program's dropouts: int64 [seed, step] on the device.  The program adds 1
    to the step after each backward pass; a captured graph reads it at each replay."""
    return torch.tensor([seed, step], dtype=torch.int64, device=device)


def dropout_threshold(p: float) -> int:
    """2^16 times the probability of a zero; raises where that is not 0 to 65535."""
    if not 0.0 <= p < 1.0 or int(p * 65536 + 0.5) > 65535:
        raise ValueError(f"p: a probability below 1 - 2^-17, not {p}")
    return int(p * 65536 + 0.5)


def _dropout_setup(x, rng, p, site, residual):
    key = ("dropout", x.shape, x.dtype, x.device, _sig(rng), p, site, _sig(residual))
    plan = _plans.get(key)
    if plan is not None:
        return plan
    _on_gpu(x, "x")
    code = _code(x, "x")
    threshold = dropout_threshold(p)
    if not 0 <= site < 1 << 32:
        raise ValueError(f"site: 0 to 2^32 - 1, not {site}")
    _like("rng", rng, x, (2,), torch.int64)
    if residual is not None:
        _like("residual", residual, x, x.shape)
    cfg = QdsDropoutConfig(ABI_VERSION, code, x.numel(), threshold, site)
    return _remember(key, (cfg, C.byref(cfg)))


def dropout_forward(x, rng, p: float, site: int = 0, residual=None):
    """y = residual + (x / (1 - p) where kept, else 0), without `residual` the latter alone.
    Which elements are kept (each with probability 1 - p, in steps of 2^-16) follows from `rng`
    (dropout_rng), `site` (a number for each dropout of a program) and the element's place in x
    alone; no mask is stored."""
    _, cfg = _dropout_setup(x, rng, p, site, residual)
    x, residual, rng = x.contiguous(), _dense(residual), rng.contiguous()
    y = x.new_empty(x.shape)
    with _on(x):
        _check(lib().qds_dropout(cfg, x.data_ptr(), _ptr(residual), rng.data_ptr(), y.data_ptr(), _stream(x)),
               "qds_dropout")
    return y


def dropout_backward(dy, rng, p: float, site: int = 0):
    """The gradient of x from that of y, with the forward call's rng, p and site (the residual's
    gradient is dy)."""
    return dropout_forward(dy, rng, p, site)


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

    class CausalConv(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, state, lengths, silu):
            y, last = causal_conv_forward(x, weight, bias, state, lengths, silu)
            ctx.save_for_backward(x, weight, bias, state, lengths)
            ctx.silu = silu
            ctx.set_materialize_grads(False)
            return y, last

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy, dlast):
            x, weight, bias, state, lengths = ctx.saved_tensors
            if dy is None:
                dy = torch.zeros_like(x)
            dx, dw, db, dfirst = causal_conv_backward(dy, x, weight, bias, state, dlast, lengths, ctx.silu)
            return dx, dw, db, None if state is None else dfirst, None, None

    class SelectiveScan(torch.autograd.Function):
        @staticmethod
        def forward(ctx, u, delta, a, b, c, skip, gate, bias, state, lengths, keep):
            o, last, marks = selective_scan_forward(u, delta, a, b, c, skip, gate, bias, state, lengths, keep)
            ctx.save_for_backward(u, delta, a, b, c, skip, gate, bias, lengths, marks)
            ctx.has_state = state is not None
            ctx.set_materialize_grads(False)
            return o, last

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, do, dlast):
            u, delta, a, b, c, skip, gate, bias, lengths, marks = ctx.saved_tensors
            if do is None:
                do = torch.zeros_like(u)
            du, ddelta, da, db, dc, dskip, dgate, dbias, dfirst = selective_scan_backward(
                do, u, delta, a, b, c, marks, skip, gate, bias, dlast, lengths)
            return du, ddelta, da, db, dc, dskip, dgate, dbias, dfirst if ctx.has_state else None, None, None

    class BranchNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, gate, residual, branch_weight, weight, residual_scale, eps):
            y, h, rstds = branch_norm_forward(x, gate, residual, branch_weight, weight, residual_scale, eps)
            ctx.save_for_backward(x, gate, residual, rstds, branch_weight, weight)
            ctx.residual_scale = residual_scale
            ctx.set_materialize_grads(False)
            return y, h

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy, dh):
            x, gate, residual, rstds, branch_weight, weight = ctx.saved_tensors
            if dy is None:
                dy = torch.zeros_like(x)
            return (*branch_norm_backward(dy, dh, x, gate, residual, rstds, branch_weight, weight,
                                          ctx.residual_scale), None, None)

    class Dropout(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, rng, p, site, residual):
            ctx.save_for_backward(rng)
            ctx.how = (p, site, residual is not None)
            return dropout_forward(x, rng, p, site, residual)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            (rng,) = ctx.saved_tensors            # raises where the program has changed it since
            p, site, has_residual = ctx.how
            dx = dropout_backward(dy, rng, p, site) if ctx.needs_input_grad[0] else None
            return dx, None, None, None, dy if has_residual else None

    _functions = (ResidualNorm, WindowAttention, DecayAttention, CausalConv, SelectiveScan, BranchNorm, Dropout)
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


def causal_conv(x, weight, bias=None, state=None, lengths=None, silu: bool = True):
    """causal_conv_forward under autograd: returns y and the last state."""
    return _autograd()[3].apply(x, weight, bias, state, lengths, silu)


def selective_scan(u, delta, a, b, c, skip=None, gate=None, bias=None, state=None, lengths=None):
    """selective_scan_forward under autograd: returns o and the last state."""
    inputs = u, delta, a, b, c, skip, gate, bias, state
    keep = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs)     # else no backward pass
    return _autograd()[4].apply(*inputs, lengths, keep)


def branch_norm(x, gate, residual, branch_weight, weight, residual_scale: float = 1.0, eps: float = 1e-6):
    """branch_norm_forward under autograd: returns y and h."""
    return _autograd()[5].apply(x, gate, residual, branch_weight, weight, residual_scale, eps)


def dropout(x, rng, p: float, site: int = 0, residual=None):
    """dropout_forward under autograd: returns y.  `rng` has to be unchanged until the backward
    pass is done (a changed one raises)."""
    return _autograd()[6].apply(x, rng, p, site, residual)
