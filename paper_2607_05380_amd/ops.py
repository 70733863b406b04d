"""Operators of a student network: binding of the handle-free calls of libtabpack.so.

An ensemble answers with a forward pass of each of its members; a student is one network trained on the ensemble's
class probabilities and served in 8 bits.  Its parts:

  distill_topk                        the loss against a teacher's top logits and its gradient
  add_rms_norm, rms_norm_backward     root-mean-square norm of x + residual, and its gradients
  gated_ff, gated_ff_backward         y = (act(x Wg^T) * (x Wu^T)) Wd^T (+ residual), and its gradients
  q8_matmul                           product of 8-bit codes with scales per row and output, optionally gated
  add_rms_norm_q8, quantize_rows      the norm, or plain rows, as 8-bit codes with a scale per row

Matrices are 2-D device tensors in bfloat16 or float32 whose rows are contiguous (any row stride and alignment).
Every call runs HIP kernels on the current stream of the tensors' device; ``PackError`` says what an argument
breaks.  Nothing is recorded for autograd: gradients come from the backward calls, and under grad mode a tensor that
requires a gradient is refused (``torch.no_grad()``, or the inside of an ``autograd.Function``, takes it).  Formulas and rules for empty, masked and non-finite rows are in ``include/tabpack.h``.
"""
import ctypes
import functools

import torch

from . import tabpack
from .tabpack import PackError

_PREC = {torch.bfloat16: 0, torch.float32: 1}

# The current stream's handle without a Stream object around it (a microsecond of a call's ten), where torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _fail(msg):
    raise PackError(msg)


def _matrix(t, name, dtype=None, shape=None):
    """Checks a 2-D device tensor with contiguous rows; its (address, row stride)."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2):
        _fail(f"{name} must be a 2-D device tensor")
    if dtype is not None and t.dtype != dtype:
        _fail(f"{name} must be {dtype}, not {t.dtype}")
    rows, cols = t.shape
    if shape is not None and (rows, cols) != shape:
        _fail(f"{name} must have shape {shape}, not {(rows, cols)}")
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        _fail(f"{name} must have contiguous rows")
    if ld < cols:
        if rows > 1:
            _fail(f"{name} must not have overlapping rows")
        ld = cols
    return t.data_ptr(), ld


def _vector(t, name, n, dtype=torch.float32):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.shape == (n,) and t.is_contiguous()):
        _fail(f"{name} must be a contiguous device tensor of {n} {dtype}")
    return t.data_ptr()


def _prec(t, name):
    if not isinstance(t, torch.Tensor) or t.dtype not in _PREC:
        _fail(f"{name} must be a bfloat16 or float32 tensor")
    return _PREC[t.dtype]


def _call(fn, like, others, *args):
    """The library call on the current stream of like's device (where all of others must be)."""
    dev = like.get_device()
    grad = torch.is_grad_enabled()
    lost = grad and like.requires_grad
    for t in others:
        if t is not None:
            if t.get_device() != dev:
                _fail("all tensors must be on one device")
            lost = lost or grad and t.requires_grad
    if lost:
        _fail("a tensor requires a gradient, which the operators do not record: call them under torch.no_grad() and "
              "take gradients from their backward calls")
    call = getattr(tabpack.load_library(), fn)
    if dev == torch.cuda.current_device():
        rc = call(*args, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = call(*args, _raw_stream(dev))
    if rc:
        tabpack._check(rc)


@functools.lru_cache(maxsize=256)
def _bytes(fn, *args):
    """A workspace size (it depends on the sizes alone)."""
    n = ctypes.c_size_t()
    tabpack._check(getattr(tabpack.load_library(), fn)(*args, ctypes.byref(n)))
    return n.value


def _empty(like, *shape, dtype=None):
    return like.new_empty(shape, dtype=dtype)


def _norm_inputs(x, weight, residual):
    prec = _prec(x, "x")
    xp, ldx = _matrix(x, "x")
    rows, cols = x.shape
    rp, ldr = (None, 0) if residual is None else _matrix(residual, "residual", x.dtype, x.shape)
    return (xp, ldx, rp, ldr, _vector(weight, "weight", cols), prec, rows, cols)


def add_rms_norm(x, weight, residual=None, eps=1e-6):
    """(y, v, rstd): v = x + residual (x itself without one), rstd = (mean v^2 + eps)^(-1/2) per row, y = v rstd weight.
    x, residual [rows, cols], weight fp32 [cols]; y and v in x's type, rstd fp32 [rows]."""
    a = _norm_inputs(x, weight, residual)
    v = x if residual is None else _empty(x, *x.shape)
    y, rstd = _empty(x, *x.shape), _empty(x, x.shape[0], dtype=torch.float32)
    _call("pack_add_rms_norm", x, (weight, residual), *a, float(eps), None if residual is None else v.data_ptr(),
          a[7], y.data_ptr(), a[7], rstd.data_ptr())
    return y, v, rstd


def add_rms_norm_q8(x, weight, residual=None, eps=1e-6):
    """(q, scale, v): add_rms_norm's y as 8-bit codes q (int8 [rows, cols]) and a scale per row (fp32 [rows]);
    y is q * scale[:, None]."""
    a = _norm_inputs(x, weight, residual)
    v = x if residual is None else _empty(x, *x.shape)
    q, scale = _empty(x, *x.shape, dtype=torch.int8), _empty(x, x.shape[0], dtype=torch.float32)
    _call("pack_add_rms_norm_q8", x, (weight, residual), *a, float(eps), None if residual is None else v.data_ptr(),
          a[7], q.data_ptr(), a[7], scale.data_ptr())
    return q, scale, v


def rms_norm_backward(dy, v, weight, rstd, dv=None):
    """(dx, dweight) of add_rms_norm: dx is the gradient of x and of the residual, dv the gradient that reaches the
    sum v on its other path (None: none).  dx in v's type, dweight fp32."""
    prec = _prec(v, "v")
    vp, ldv = _matrix(v, "v")
    yp, ldy = _matrix(dy, "dy", v.dtype, v.shape)
    rows, cols = v.shape
    dp, ldd = (None, 0) if dv is None else _matrix(dv, "dv", v.dtype, v.shape)
    wp, rp = _vector(weight, "weight", cols), _vector(rstd, "rstd", rows)
    dx, dw = _empty(v, rows, cols), _empty(v, cols, dtype=torch.float32)
    work = _empty(v, _bytes("pack_rms_norm_backward_workspace_size", rows, cols), dtype=torch.uint8)
    _call("pack_rms_norm_backward", v, (dy, weight, rstd, dv), yp, ldy, vp, ldv, wp, rp, dp, ldd, prec, rows, cols,
          dx.data_ptr(), cols, dw.data_ptr(), work.data_ptr(), work.numel())
    return dx, dw


def quantize_rows(x):
    """(q, scale): rows as 8-bit codes with a scale each; x is about q * scale[:, None]."""
    prec = _prec(x, "x")
    xp, ldx = _matrix(x, "x")
    rows, cols = x.shape
    q, scale = _empty(x, rows, cols, dtype=torch.int8), _empty(x, rows, dtype=torch.float32)
    _call("pack_quantize_rows", x, (), xp, ldx, prec, rows, cols, q.data_ptr(), cols, scale.data_ptr())
    return q, scale


def distill_topk(logits, idx, teacher, temperature=1.0, row_weight=None, grad=True):
    """(loss, grad): the distillation loss of each row against its teacher entries and its gradient.

    logits [rows, classes]; idx int32 and teacher fp32 [rows, k]: classes and logits of the teacher's entries (a
    negative index or a logit of -inf: left out); row_weight fp32 [rows]: the factor of each row's loss in the
    caller's total (None: 1).  loss fp32 [rows]; grad in logits' type, or None with grad=False."""
    prec = _prec(logits, "logits")
    zp, ldz = _matrix(logits, "logits")
    rows, classes = logits.shape
    _matrix(idx, "idx", torch.int32)
    k = idx.shape[1]
    if k >= 1 << 31:  # (the C call counts in 32 bits; of the sizes this one alone is no leading dimension)
        _fail(f"k={k} must be below 2^31")
    if idx.shape[0] != rows:
        _fail(f"idx must have {rows} rows, not {idx.shape[0]}")
    _matrix(teacher, "teacher", torch.float32, (rows, k))
    if not (idx.is_contiguous() and teacher.is_contiguous()):
        _fail("idx and teacher must be contiguous")
    wp = None if row_weight is None else _vector(row_weight, "row_weight", rows)
    loss = _empty(logits, rows, dtype=torch.float32)
    g = _empty(logits, rows, classes) if grad else None
    _call("pack_distill_topk", logits, (idx, teacher, row_weight), zp, ldz, prec, rows, classes, idx.data_ptr(),
          teacher.data_ptr(), k, float(temperature), wp, loss.data_ptr(), g.data_ptr() if grad else None, classes)
    return loss, g


def _act(act):
    if act not in tabpack.ACTIVATIONS:
        _fail(f"unknown activation {act!r}")
    return tabpack.ACTIVATIONS[act]


def _work(like, fn, *args):
    n = _bytes(fn, *args)
    return _empty(like, n, dtype=torch.uint8) if n else None


def _ff_inputs(x, w_gate_up, w_down):
    prec = _prec(x, "x")
    xp, ldx = _matrix(x, "x")
    tokens, d_in = x.shape
    wdp, ldwd = _matrix(w_down, "w_down", x.dtype)
    d_out, hidden = w_down.shape
    wgp, ldwg = _matrix(w_gate_up, "w_gate_up", x.dtype, (2 * hidden, d_in))
    return prec, (tokens, d_in, hidden, d_out), (xp, ldx, wgp, ldwg, wdp, ldwd)


def _ff_ld(x, cols):
    """Elements from row to row of the hidden values and of the gradients of gate and up (see tabpack.h)."""
    return (cols + 7) // 8 * 8 if x.dtype is torch.bfloat16 else (cols + 3) // 4 * 4


def gated_ff(x, w_gate_up, w_down, act="silu", residual=None, save=False):
    """y = h w_down^T (+ residual) with [g | u] = x w_gate_up^T and h = act(g) u: x [tokens, d_in], w_gate_up
    [2 hidden, d_in] (gate rows, then up rows), w_down [d_out, hidden], all in one type; act "silu", "gelu" or
    "relu".  save=True: (y, saved), saved = ([g | u] in fp32, h) for gated_ff_backward."""
    prec, dims, ptrs = _ff_inputs(x, w_gate_up, w_down)
    tokens, _, hidden, d_out = dims
    rp, ldr = (None, 0) if residual is None else _matrix(residual, "residual", x.dtype, (tokens, d_out))
    code = _act(act)
    gu = _empty(x, tokens, 2 * hidden, dtype=torch.float32) if save else None
    h, y = _empty(x, tokens, _ff_ld(x, hidden)), _empty(x, tokens, d_out)
    work = _work(x, "pack_gated_ff_workspace_size", prec, *dims, 0)
    _call("pack_gated_ff_forward", x, (w_gate_up, w_down, residual), *ptrs, rp, ldr, prec, code, *dims,
          gu.data_ptr() if save else None, h.data_ptr(), y.data_ptr(), d_out,
          None if work is None else work.data_ptr(), 0 if work is None else work.numel())
    return (y, (gu, h[:, :hidden])) if save else y


def gated_ff_backward(dy, x, w_gate_up, w_down, saved, act="silu", need_dx=True):
    """(dx, dw_gate_up, dw_down) of gated_ff from dy [tokens, d_out] and what it saved (the residual's gradient is
    dy itself), in x's type; dx is None with need_dx=False."""
    prec, dims, ptrs = _ff_inputs(x, w_gate_up, w_down)
    tokens, d_in, hidden, d_out = dims
    gp, ldg = _matrix(dy, "dy", x.dtype, (tokens, d_out))
    gu, h = saved
    _matrix(gu, "saved gate and up values", torch.float32, (tokens, 2 * hidden))
    _matrix(h, "saved hidden values", x.dtype, (tokens, hidden))
    if not gu.is_contiguous():
        _fail("saved gate and up values must be contiguous")
    code = _act(act)
    ldh = _ff_ld(x, hidden)
    if h.stride(0) != ldh or (ldh > hidden and h.untyped_storage().nbytes() <
                              (h.storage_offset() + tokens * ldh) * h.element_size()):
        own = _empty(x, tokens, ldh)  # (a copy of what gated_ff saved, in rows of another length)
        own[:, :hidden] = h
        h = own
    dgu = _empty(x, tokens, _ff_ld(x, 2 * hidden))
    dx = _empty(x, tokens, d_in) if need_dx else None
    dwg, dwd = _empty(x, 2 * hidden, d_in), _empty(x, d_out, hidden)
    work = _work(x, "pack_gated_ff_workspace_size", prec, *dims, 1)
    _call("pack_gated_ff_backward", x, (dy, w_gate_up, w_down, gu, h), gp, ldg, *ptrs, gu.data_ptr(), h.data_ptr(),
          prec, code, *dims, dgu.data_ptr(), dx.data_ptr() if need_dx else None, d_in, dwg.data_ptr(), dwd.data_ptr(),
          None if work is None else work.data_ptr(), 0 if work is None else work.numel())
    return dx, dwg, dwd


def q8_matmul(q, scale, w, w_scale, bias=None, gate=None, dtype=torch.bfloat16):
    """(q * scale[:, None]) (w * w_scale[:, None])^T (+ bias) of 8-bit codes q int8 [rows, depth] and w int8
    [outputs, depth], scales and bias fp32, summed exactly in int32; [rows, outputs] in ``dtype``.  gate: an activation
    name; w, w_scale and bias then hold the gate rows and the up rows, and the result is act(gate) * up."""
    qp, ldq = _matrix(q, "q", torch.int8)
    rows, depth = q.shape
    wp, ldw = _matrix(w, "w", torch.int8)
    n = w.shape[0]
    if w.shape[1] != depth:
        _fail(f"w must have {depth} columns, not {w.shape[1]}")
    code = -1 if gate is None else _act(gate)
    if gate is not None and n % 2:
        _fail("a gated w holds as many gate rows as up rows")
    if dtype not in _PREC:
        _fail("dtype must be bfloat16 or float32")
    sp, wsp = _vector(scale, "scale", rows), _vector(w_scale, "w_scale", n)
    bp = None if bias is None else _vector(bias, "bias", n)
    outputs = n if gate is None else n // 2
    out = _empty(q, rows, outputs, dtype=dtype)
    work = _work(q, "pack_q8_matmul_workspace_size", rows, outputs, depth, code)
    _call("pack_q8_matmul", q, (scale, w, w_scale, bias), qp, ldq, sp, wp, ldw, wsp, bp, code, _PREC[dtype], rows,
          outputs, depth, out.data_ptr(), outputs, None if work is None else work.data_ptr(),
          0 if work is None else work.numel())
    return out
