"""ctypes binding of the operators around the attention and the scan (``include/fla_seq.h``).

Argument marshalling only, as in ``binding``: every step runs inside ``libfla_seq.so``.  The ``fla_*``
functions mirror the C ABI on tensors or raw device addresses.  The tensor-level functions check types,
shapes and layouts, allocate what they return, and launch on ``stream`` (default: the current stream of
the tensors' device, which need not be the current device); with a ``stream`` given, what they allocate
belongs to that stream.
"""
from __future__ import annotations

import ctypes
import functools
import os

from .binding import FlaError, _check, _lock, _ptr, _stream

FLA_F32, FLA_BF16 = 0, 1
ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}

_LIB_NAME = "libfla_seq.so"
_lib = None


def seq_library_path() -> str:
    return os.path.join(os.path.dirname(os.path.abspath(__file__)), _LIB_NAME)


def _declare(lib):
    P, I, Z, L, F, D = (ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_int64, ctypes.c_float,
                        ctypes.c_double)
    size = ctypes.POINTER(Z)
    for name, args in {
        "fla_add_rms_norm_fwd": [P, L, P, L, P, P, P, P, L, I, F, I, I, P],
        "fla_add_rms_norm_q8": [P, L, P, L, P, P, P, P, L, I, I, F, I, I, P],
        "fla_add_rms_norm_bwd_workspace": [L, I, size],
        "fla_add_rms_norm_bwd": [P, L, P, L, P, P, P, L, P, P, P, Z, L, I, I, I, P],
        "fla_rotary": [P, L, L, L] * 4 + [P, I, L, L, I, P, I, I, I, I, I, I, I, D, I, I, P],
        "fla_rotary_freqs": [I, D, I, D, D, P, ctypes.POINTER(D)],
        "fla_gated_scan_states": [I, I, I, size],
        "fla_gated_scan_workspace": [I, I, I, size],
        "fla_gated_scan_bwd_workspace": [I, I, I, size],
        "fla_gated_scan_fwd": [P, L, L] * 3 + [P, P, P, P, P, P, P, Z, I, I, I, F, I, P],
        "fla_gated_scan_bwd": [P, L, L] * 3 + [P, P, P, P, L, L, P, P, P, P, P, P, P, Z, I, I, I, F, I, P],
    }.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, I


def load_seq_library():
    """Load (once) and return the ctypes handle of libfla_seq.so."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            path = seq_library_path()
            if not os.path.exists(path):
                raise FlaError(-1, "%s is not built; run __graft_entry__.build()" % path)
            lib = ctypes.CDLL(path)
            _declare(lib)
            _lib = lib
    return _lib


def _done(rc, check=True):
    if rc != 0 and check:
        _check(rc)
    return rc


def _at(t):
    """A tensor's address, or None."""
    return None if t is None else t.data_ptr()


def _size(fn, *args) -> int:
    n = ctypes.c_size_t()
    _check(fn(*args, ctypes.byref(n)))
    return n.value


# ---- the C ABI -------------------------------------------------------------------------------

def fla_add_rms_norm_fwd(x, x_stride, residual, residual_stride, weight, y, sum, rstd, rows, D, eps, dtype,
                         weight_dtype, stream=None, check=True) -> int:
    """y = rms_norm(x + residual) * weight, the sum and 1 / rms.  Tensors or raw addresses."""
    return _done(load_seq_library().fla_add_rms_norm_fwd(
        _ptr(x), x_stride, _ptr(residual), residual_stride, _ptr(weight), _ptr(y), _ptr(sum), _ptr(rstd), rows, D, eps,
        dtype, weight_dtype, _stream(stream)), check)


def fla_add_rms_norm_q8(x, x_stride, residual, residual_stride, weight, q, scales, sum, rows, D, group, eps, dtype,
                        weight_dtype, stream=None, check=True) -> int:
    """The same with e4m3 output and scales."""
    return _done(load_seq_library().fla_add_rms_norm_q8(
        _ptr(x), x_stride, _ptr(residual), residual_stride, _ptr(weight), _ptr(q), _ptr(scales), _ptr(sum), rows, D,
        group, eps, dtype, weight_dtype, _stream(stream)), check)


@functools.lru_cache(maxsize=1024, typed=True)   # a function of the sizes alone
def fla_add_rms_norm_bwd_workspace(rows, D) -> int:
    return _size(load_seq_library().fla_add_rms_norm_bwd_workspace, rows, D)


def fla_add_rms_norm_bwd(dy, dy_stride, s, s_stride, weight, rstd, dsum, dsum_stride, dx, dweight, workspace,
                         workspace_bytes, rows, D, dtype, weight_dtype, stream=None, check=True) -> int:
    """Gradients of the norm at the sum s."""
    return _done(load_seq_library().fla_add_rms_norm_bwd(
        _ptr(dy), dy_stride, _ptr(s), s_stride, _ptr(weight), _ptr(rstd), _ptr(dsum), dsum_stride, _ptr(dx),
        _ptr(dweight), _ptr(workspace), workspace_bytes, rows, D, dtype, weight_dtype, _stream(stream)), check)


def fla_rotary_freqs(rot, theta=10000.0, scaling=0, factor=1.0, trained_len=1.0):
    """(list of rot / 2 frequencies, mscale), computed by the library on the host."""
    out, m = (ctypes.c_double * max(rot // 2, 1))(), ctypes.c_double()
    _check(load_seq_library().fla_rotary_freqs(rot, theta, scaling, factor, trained_len, out, ctypes.byref(m)))
    return list(out), m.value


def fla_rotary(q, q_strides, k, k_strides, q_out, qo_strides, k_out, ko_strides, positions, pos64, pos_batch,
               pos_token, axes, freqs, B, L, hq, hk, d, rot, interleaved, mscale=1.0, inverse=0, dtype=FLA_BF16,
               stream=None, check=True) -> int:
    """Rotation of q and k; *_strides: (batch, token, head) in elements."""
    return _done(load_seq_library().fla_rotary(
        _ptr(q), *q_strides, _ptr(k), *k_strides, _ptr(q_out), *qo_strides, _ptr(k_out), *ko_strides, _ptr(positions),
        pos64, pos_batch, pos_token, axes, _ptr(freqs), B, L, hq, hk, d, rot, interleaved, mscale, inverse, dtype,
        _stream(stream)), check)


@functools.lru_cache(maxsize=1024, typed=True)   # a function of the sizes alone
def fla_gated_scan_states(B, L, D) -> int:
    return _size(load_seq_library().fla_gated_scan_states, B, L, D)


@functools.lru_cache(maxsize=1024, typed=True)   # a function of the sizes alone
def fla_gated_scan_workspace(B, L, D) -> int:
    return _size(load_seq_library().fla_gated_scan_workspace, B, L, D)


@functools.lru_cache(maxsize=1024, typed=True)   # a function of the sizes alone
def fla_gated_scan_bwd_workspace(B, L, D) -> int:
    return _size(load_seq_library().fla_gated_scan_bwd_workspace, B, L, D)


def fla_gated_scan_fwd(x, x_strides, r, r_strides, i, i_strides, lam, h0, lengths, h, h_last, states, workspace,
                       workspace_bytes, B, L, D, c=8.0, dtype=FLA_BF16, stream=None, check=True) -> int:
    """The recurrence; *_strides: (batch, token) in elements."""
    return _done(load_seq_library().fla_gated_scan_fwd(
        _ptr(x), *x_strides, _ptr(r), *r_strides, _ptr(i), *i_strides, _ptr(lam), _ptr(h0), _ptr(lengths), _ptr(h),
        _ptr(h_last), _ptr(states), _ptr(workspace), workspace_bytes, B, L, D, c, dtype, _stream(stream)), check)


def fla_gated_scan_bwd(x, x_strides, r, r_strides, i, i_strides, lam, states, lengths, dh, dh_strides, d_last, dx, dr,
                       di, dlam, dh0, workspace, workspace_bytes, B, L, D, c=8.0, dtype=FLA_BF16, stream=None,
                       check=True) -> int:
    """Its gradients."""
    return _done(load_seq_library().fla_gated_scan_bwd(
        _ptr(x), *x_strides, _ptr(r), *r_strides, _ptr(i), *i_strides, _ptr(lam), _ptr(states), _ptr(lengths),
        _ptr(dh), *dh_strides, _ptr(d_last), _ptr(dx), _ptr(dr), _ptr(di), _ptr(dlam), _ptr(dh0), _ptr(workspace),
        workspace_bytes, B, L, D, c, dtype, _stream(stream)), check)


# ---- tensors -------------------------------------------------------------------------------------

_codes = {}


def _dtype(t):
    code = _codes.get(t.dtype)
    if code is None:
        import torch
        _codes.update({torch.float32: FLA_F32, torch.bfloat16: FLA_BF16})
        code = _codes.get(t.dtype)
        if code is None:
            raise TypeError("tensors must be bfloat16 or float32, got %s" % t.dtype)
    return code


def _on(t, stream, body):
    """body(raw stream) with t's device current, on `stream` or that device's current one."""
    import torch
    device = t.device
    if device.type != "cuda":
        raise ValueError("tensors must be on the GPU")
    if stream is None:
        if device.index == torch.cuda.current_device():
            return body(torch._C._cuda_getCurrentRawStream(device.index))
        with torch.cuda.device(device):
            return body(torch._C._cuda_getCurrentRawStream(device.index))
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
    if stream.device != device:
        raise ValueError("the stream is on %s, the tensors on %s" % (stream.device, device))
    with torch.cuda.stream(stream):
        return body(stream.cuda_stream)


def _new(like):
    """A contiguous tensor of like's shape and type."""
    import torch
    return torch.empty_like(like, memory_format=torch.contiguous_format)


def _same(name, t, like, shape, dtype=None):
    """t on like's device, of this shape and type (default: like's)."""
    if dtype is None:
        dtype = like.dtype
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.device != like.device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, like.device))
    if t.shape != shape:   # (a torch.Size compares as a tuple)
        raise ValueError("%s must be %s, got %s" % (name, tuple(shape), tuple(t.shape)))


def _whole(name, t, like, shape, dtype=None):
    """The same, and contiguous."""
    _same(name, t, like, shape, dtype)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _rows(name, t):
    """Elements between the rows of a [..., D] tensor with contiguous channels and evenly spaced rows."""
    if t.dim() == 0:
        raise ValueError("%s must have channels" % name)
    if t.is_contiguous() or t.numel() == 0:
        return t.shape[-1]
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("%s must have contiguous channels" % name)
    step = None
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n == 1:
            continue
        if step is None:
            step, period = s, s * n
        elif s != period:
            raise ValueError("%s must have evenly spaced rows" % name)
        else:
            period = s * n
    return t.shape[-1] if step is None else step


def _strides(name, t):
    """All strides but the last, of a tensor with contiguous channels."""
    *strides, last = t.stride()
    if last != 1 and t.shape[-1] > 1 and t.numel():
        raise ValueError("%s must have contiguous channels" % name)
    return strides


def _norm_args(x, weight, residual):
    dtype = wdtype = _dtype(x)
    shape = x.shape
    stride, rstride = _rows("x", x), 0
    D = shape[-1]
    if residual is not None:
        _same("residual", residual, x, shape)
        rstride = _rows("residual", residual)
    if weight.dtype != x.dtype:
        import torch
        wdtype = FLA_F32
        _whole("weight", weight, x, (D,), torch.float32)
    else:
        _whole("weight", weight, x, (D,))
    return dtype, wdtype, x.numel() // D if D else 0, D, stride, rstride


def _norm_fwd(x, weight, residual, eps, out, sum_out, keep, stream):
    import torch
    dtype, wdtype, rows, D, stride, rstride = _norm_args(x, weight, residual)
    if out is not None:
        _whole("out", out, x, x.shape)
    if sum_out is not None:
        _whole("sum_out", sum_out, x, x.shape)

    def body(raw):
        y = _new(x) if out is None else out
        s = sum_out
        if s is None and residual is not None:
            s = _new(x)
        rstd = x.new_empty(x.shape[:-1], dtype=torch.float32) if keep else None
        _done(load_seq_library().fla_add_rms_norm_fwd(
            x.data_ptr(), stride, _at(residual), rstride, weight.data_ptr(), y.data_ptr(), _at(s), _at(rstd), rows, D, eps,
            dtype, wdtype, raw))
        return y, x if s is None else s, rstd

    return _on(x, stream, body)


def add_rms_norm(x, weight, residual=None, eps=1e-6, out=None, sum_out=None, stream=None):
    """Root-mean-square norm of s = x + residual over the last dimension, times weight: (y, s).

    x, residual: [..., D], bf16 or fp32, contiguous channels and evenly spaced rows; weight [D] of x's
    type or fp32.  s is rounded to x's type (the norm takes it unrounded); without a residual it is x
    itself.  out and sum_out (contiguous) may be x or residual: in place."""
    return _norm_fwd(x, weight, residual, eps, out, sum_out, False, stream)[:2]


def add_rms_norm_fwd_train(x, weight, residual=None, eps=1e-6, stream=None):
    """The same, and 1 / rms of each row for the backward: (y, s, rstd)."""
    return _norm_fwd(x, weight, residual, eps, None, None, True, stream)


def add_rms_norm_q8(x, weight, residual=None, eps=1e-6, group=0, sum_out=None, stream=None):
    """The same with y in 8 bits: (q, scales, s), y ~ q * scales.  q: float8_e4m3fn of x's shape;
    scales: fp32 [..., ceil(D / group)] for groups of 32, 64 or 128 channels, [..., 1] for group = 0 (a
    scale for each row)."""
    import torch
    dtype, wdtype, rows, D, stride, rstride = _norm_args(x, weight, residual)
    if sum_out is not None:
        _whole("sum_out", sum_out, x, x.shape)
    if group not in (0, 32, 64, 128):
        raise ValueError("group must be 0, 32, 64 or 128, got %r" % (group,))

    def body(raw):
        q = x.new_empty(x.shape, dtype=torch.float8_e4m3fn)
        scales = x.new_empty((*x.shape[:-1], -(-D // group) if group else 1), dtype=torch.float32)
        s = sum_out
        if s is None and residual is not None:
            s = _new(x)
        _done(load_seq_library().fla_add_rms_norm_q8(
            x.data_ptr(), stride, _at(residual), rstride, weight.data_ptr(), q.data_ptr(), scales.data_ptr(), _at(s), rows,
            D, group, eps, dtype, wdtype, raw))
        return q, scales, x if s is None else s

    return _on(x, stream, body)


def add_rms_norm_bwd(dy, s, weight, rstd, dsum=None, stream=None):
    """Gradients of add_rms_norm at the sum s: (dx, dweight).  dx is that of x and of residual alike;
    dsum: the gradient that reaches s from behind (None: none).  dweight is fp32."""
    import torch
    dtype, wdtype, rows, D, stride, dystride = _norm_args(s, weight, dy)
    _whole("rstd", rstd, s, s.shape[:-1], torch.float32)
    dsstride = 0
    if dsum is not None:
        _same("dsum", dsum, s, s.shape)
        dsstride = _rows("dsum", dsum)

    def body(raw):
        dx = _new(s)
        nbytes = fla_add_rms_norm_bwd_workspace(rows, D)
        dw, ws = rstd.new_empty(D), rstd.new_empty(nbytes // 4)
        _done(load_seq_library().fla_add_rms_norm_bwd(
            dy.data_ptr(), dystride, s.data_ptr(), stride, weight.data_ptr(), rstd.data_ptr(), _at(dsum), dsstride,
            dx.data_ptr(), dw.data_ptr(), ws.data_ptr(), nbytes, rows, D, dtype, wdtype, raw))
        return dx, dw

    return _on(s, stream, body)


def rotary_freqs(rot, theta=10000.0, scaling="none", factor=1.0, trained_len=4096.0, axes=1, device="cuda"):
    """(freqs, mscale) for ``rotary``: float64 [rot / 2] on the device, and the factor on the rotated
    vectors.  scaling for contexts `factor` times longer than the trained one: "none", "linear" (positions
    interpolated), "base" (a larger theta) or "parts" (slow pairs interpolated, fast ones kept).  axes = 2:
    each axis turns half of the pairs, with the frequencies of rot / 2 channels."""
    import torch
    if scaling not in ROPE_SCALINGS:
        raise ValueError("scaling must be one of %s, got %r" % (sorted(ROPE_SCALINGS), scaling))
    if axes not in (1, 2) or rot % (2 * axes):
        raise ValueError("%d channels do not divide into pairs of %d axes" % (rot, axes))
    f, mscale = fla_rotary_freqs(rot // axes, float(theta), ROPE_SCALINGS[scaling], float(factor), float(trained_len))
    return torch.tensor(f * axes, dtype=torch.float64, device=device), mscale


def _rotary(q, k, freqs, positions, interleaved, mscale, out, inverse, stream):
    import torch
    dtype = _dtype(q)
    if q.dim() != 4:
        raise ValueError("q must be [B, L, heads, d], got %s" % (tuple(q.shape),))
    B, L, hq, d = q.shape
    hk, kstr = 0, (0, 0, 0)
    if k is not None:
        if k.dim() != 4:
            raise ValueError("k must be [B, L, heads, d], got %s" % (tuple(k.shape),))
        hk = k.shape[2]
        _same("k", k, q, (B, L, hk, d))
        kstr = _strides("k", k)
    if positions.dtype not in (torch.int32, torch.int64):
        raise TypeError("positions must be int32 or int64, got %s" % positions.dtype)
    axes = 1
    if positions.dim() == 3:
        axes = 2
        _same("positions", positions, q, (B, L, 2), positions.dtype)
        if positions.stride(2) != 1 and positions.numel():
            raise ValueError("positions must have their axes side by side")
    else:
        _same("positions", positions, q, (B, L), positions.dtype)
    if freqs.dim() != 1:
        raise ValueError("freqs must be [rot / 2], got %s" % (tuple(freqs.shape),))
    _whole("freqs", freqs, q, freqs.shape, torch.float64)
    qstr = _strides("q", q)
    qo, ko = (None, None) if out is None else out
    if qo is not None:
        _same("out[0]", qo, q, q.shape)
    if ko is not None:
        if k is None:
            raise ValueError("out[1] without k")
        _same("out[1]", ko, k, k.shape)

    def body(raw):
        qr = _new(q) if qo is None else qo
        kr = ko
        if kr is None and k is not None:
            kr = _new(k)
        _done(load_seq_library().fla_rotary(
            q.data_ptr(), *qstr, _at(k), *kstr, qr.data_ptr(), *_strides("out[0]", qr), _at(kr),
            *(_strides("out[1]", kr) if hk else kstr), positions.data_ptr(), positions.dtype == torch.int64,
            *positions.stride()[:2], axes, freqs.data_ptr(), B, L, hq, hk, d, 2 * freqs.shape[0], interleaved, mscale,
            inverse, dtype, raw))
        return qr, kr

    return _on(q, stream, body)


def rotary(q, k, freqs, positions, interleaved=False, mscale=1.0, out=None, stream=None):
    """Rotary positions of q [B, L, hq, d] and k [B, L, hk, d] (None: q alone): (q', k').

    freqs [rot / 2] and mscale as ``rotary_freqs`` gives them: the first rot channels of each head turn, in
    pairs (j, j + rot / 2), or (2j, 2j + 1) if interleaved; the others are copied.  positions: int32 or
    int64 [B, L], or [B, L, 2] for two axes (pairs of the first half turn with the first).  Any strides
    with contiguous channels; out = (q_out, k_out) may be (q, k): in place."""
    return _rotary(q, k, freqs, positions, interleaved, mscale, out, 0, stream)


def rotary_bwd(dq, dk, freqs, positions, interleaved=False, mscale=1.0, out=None, stream=None):
    """Gradients of ``rotary`` with respect to q and k: the rotation back, times mscale."""
    return _rotary(dq, dk, freqs, positions, interleaved, mscale, out, 1, stream)


def _scan_args(x, r, i, lam, lengths, dim=3):
    import torch
    dtype = _dtype(x)
    if x.dim() != dim:
        raise ValueError("x must be %s, got %s" % ("[B, L, D]" if dim == 3 else "[B, D]", tuple(x.shape)))
    _same("r", r, x, x.shape)
    _same("i", i, x, x.shape)
    _whole("lam", lam, x, x.shape[-1:], torch.float32)
    if lengths is not None:
        _whole("lengths", lengths, x, x.shape[:1], torch.int32)
    return dtype, (_strides("x", x), _strides("r", r), _strides("i", i))


def _scan_fwd(x, r, i, lam, h0, lengths, c, out, keep, stream):
    import torch
    dtype, (xs, rs, is_) = _scan_args(x, r, i, lam, lengths)
    B, L, D = x.shape
    if h0 is not None:
        _whole("h0", h0, x, (B, D), torch.float32)
    if out is not None:
        _whole("out", out, x, x.shape)

    def body(raw):
        h = _new(x) if out is None else out
        last = lam.new_empty((B, D))
        states = lam.new_empty(fla_gated_scan_states(B, L, D) // 4) if keep else None
        nbytes = fla_gated_scan_workspace(B, L, D)
        ws = lam.new_empty(nbytes // 4) if nbytes else None
        _done(load_seq_library().fla_gated_scan_fwd(
            x.data_ptr(), *xs, r.data_ptr(), *rs, i.data_ptr(), *is_, lam.data_ptr(), _at(h0), _at(lengths), h.data_ptr(),
            last.data_ptr(), _at(states), _at(ws), nbytes, B, L, D, c, dtype, raw))
        return h, last, states

    return _on(x, stream, body)


def gated_scan(x, r, i, lam, h0=None, lengths=None, c=8.0, out=None, stream=None):
    """Gated linear recurrence over the tokens: (h, h_last).

    x and the gates before their sigmoids r (decay), i (input): [B, L, D], bf16 or fp32, any strides with
    contiguous channels; lam [D] fp32; per channel
      a = exp(-c softplus(lam) sigmoid(r)),   h = a h_before + sqrt(1 - a^2) sigmoid(i) x
    from the state h0 ([B, D] fp32; None: 0).  h_last [B, D] fp32 is the state behind the last token.
    lengths [B] int32: tokens from there on are skipped; their rows of h keep what `out` held (without
    `out`: anything)."""
    return _scan_fwd(x, r, i, lam, h0, lengths, c, out, False, stream)[:2]


def gated_scan_fwd_train(x, r, i, lam, h0=None, lengths=None, c=8.0, out=None, stream=None):
    """The same, and the states that the backward starts its chunks from: (h, h_last, states)."""
    return _scan_fwd(x, r, i, lam, h0, lengths, c, out, True, stream)


def gated_scan_step(x, r, i, lam, state, c=8.0, out=None, new_state=None, stream=None):
    """One token: x, r, i [B, D], state [B, D] fp32: (h, new_state).  new_state may be `state`: in place."""
    import torch
    dtype, (xs, rs, is_) = _scan_args(x, r, i, lam, None, dim=2)
    B, D = x.shape
    _whole("state", state, x, (B, D), torch.float32)
    if new_state is not None:
        _whole("new_state", new_state, x, (B, D), torch.float32)
    if out is not None:
        _whole("out", out, x, (B, D))

    def body(raw):
        h = _new(x) if out is None else out
        ns = _new(state) if new_state is None else new_state
        _done(load_seq_library().fla_gated_scan_fwd(
            x.data_ptr(), xs[0], 0, r.data_ptr(), rs[0], 0, i.data_ptr(), is_[0], 0, lam.data_ptr(), state.data_ptr(), None,
            h.data_ptr(), ns.data_ptr(), None, None, 0, B, 1, D, c, dtype, raw))
        return h, ns

    return _on(x, stream, body)


def gated_scan_bwd(x, r, i, lam, states, dh, d_last=None, lengths=None, c=8.0, stream=None):
    """Gradients of gated_scan: (dx, dr, di, dlam, dh0), dlam and dh0 fp32.  states from
    gated_scan_fwd_train of the same inputs; dh [B, L, D] and d_last [B, D] fp32 may be None (zero)."""
    import torch
    dtype, (xs, rs, is_) = _scan_args(x, r, i, lam, lengths)
    B, L, D = x.shape
    _whole("states", states, x, (fla_gated_scan_states(B, L, D) // 4,), torch.float32)
    ds = (0, 0)
    if dh is not None:
        _same("dh", dh, x, x.shape)
        ds = _strides("dh", dh)
    if d_last is not None:
        _whole("d_last", d_last, x, (B, D), torch.float32)

    def body(raw):
        dx, dr, di = _new(x), _new(x), _new(x)
        nbytes = fla_gated_scan_bwd_workspace(B, L, D)
        dlam, dh0, ws = lam.new_empty(D), lam.new_empty((B, D)), lam.new_empty(nbytes // 4)
        _done(load_seq_library().fla_gated_scan_bwd(
            x.data_ptr(), *xs, r.data_ptr(), *rs, i.data_ptr(), *is_, lam.data_ptr(), states.data_ptr(), _at(lengths),
            _at(dh), *ds, _at(d_last), dx.data_ptr(), dr.data_ptr(), di.data_ptr(), dlam.data_ptr(), dh0.data_ptr(),
            ws.data_ptr(), nbytes, B, L, D, c, dtype, raw))
        return dx, dr, di, dlam, dh0

    return _on(x, stream, body)


# ---- torch autograd --------------------------------------------------------------------------

_functions = None


def _channels(t):
    """t, or a copy of it, with contiguous channels."""
    return t if t is None or t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


def _even(t):
    """t, or a copy of it, with contiguous channels and evenly spaced rows."""
    try:
        _rows("", t)
        return t
    except ValueError:
        return t.contiguous()


def _autograd():
    """The torch.autograd.Functions; built on first use so that importing the package does not import torch."""
    global _functions
    if _functions is not None:
        return _functions
    import torch
    from torch.autograd.function import once_differentiable

    class AddRmsNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, residual, eps):
            ctx.set_materialize_grads(False)
            x, residual, weight = _even(x), None if residual is None else _even(residual), weight.contiguous()
            y, s, rstd = add_rms_norm_fwd_train(x, weight, residual, eps)
            ctx.save_for_backward(s, weight, rstd)
            ctx.with_residual = residual is not None
            return (y, s) if ctx.with_residual else y

        @staticmethod
        @once_differentiable
        def backward(ctx, dy, ds=None):
            s, weight, rstd = ctx.saved_tensors
            dw = None
            if dy is None:
                dx = ds
            else:
                dx, dw = add_rms_norm_bwd(_even(dy), s, weight, rstd, None if ds is None else _even(ds))
                dw = dw.to(weight.dtype)
            return dx, dw, dx if ctx.with_residual else None, None

    class Rotary(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, freqs, positions, interleaved, mscale):
            ctx.save_for_backward(freqs, positions)
            ctx.cfg = (interleaved, mscale)
            return rotary(_channels(q), _channels(k), freqs, positions, interleaved, mscale)

        @staticmethod
        @once_differentiable
        def backward(ctx, dq, dk):
            freqs, positions = ctx.saved_tensors
            dq, dk = rotary_bwd(_channels(dq), _channels(dk), freqs, positions, *ctx.cfg)
            return dq, dk, None, None, None, None

    class GatedRecurrence(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, r, i, lam, h0, lengths, c):
            ctx.set_materialize_grads(False)
            x, r, i = _channels(x), _channels(r), _channels(i)
            lam, h0 = lam.contiguous(), None if h0 is None else h0.contiguous()
            out = None if lengths is None else torch.zeros(x.shape, dtype=x.dtype, device=x.device)
            h, last, states = gated_scan_fwd_train(x, r, i, lam, h0, lengths, c, out)
            ctx.save_for_backward(x, r, i, lam, states, lengths)
            ctx.c, ctx.with_h0 = c, h0 is not None
            return h, last

        @staticmethod
        @once_differentiable
        def backward(ctx, dh, d_last):
            if dh is None and d_last is None:
                return (None,) * 7
            x, r, i, lam, states, lengths = ctx.saved_tensors
            d_last = None if d_last is None else d_last.contiguous()
            dx, dr, di, dlam, dh0 = gated_scan_bwd(x, r, i, lam, states, _channels(dh), d_last, lengths, ctx.c)
            return dx, dr, di, dlam, dh0 if ctx.with_h0 else None, None, None

    _functions = AddRmsNorm, Rotary, GatedRecurrence
    return _functions


def residual_rms_norm(x, weight, residual=None, eps=1e-6):
    """Differentiable add_rms_norm on the current stream: (y, s); without a residual s is x.  The
    gradients are those at the sum as it is kept, rounded to x's type."""
    if residual is None:
        return _autograd()[0].apply(x, weight, None, float(eps)), x
    return _autograd()[0].apply(x, weight, residual, float(eps))


def rotary_embedding(q, k, freqs, positions, interleaved=False, mscale=1.0):
    """Differentiable rotary on the current stream: (q', k'); k may be None."""
    return _autograd()[1].apply(q, k, freqs, positions, bool(interleaved), float(mscale))


def gated_recurrence(x, r, i, lam, h0=None, lengths=None, c=8.0):
    """Differentiable gated_scan on the current stream: (h, h_last); rows of h from lengths[b] on are 0."""
    return _autograd()[2].apply(x, r, i, lam, h0, lengths, float(c))
