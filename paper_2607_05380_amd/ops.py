"""Operators of a student network: binding of the handle-free calls of libtabpack.so.

An ensemble answers with a forward pass of each of its members; a student is one network trained on the ensemble's
class probabilities and served in 8 bits.  Its parts:

  distill_topk                        the loss against a teacher's top logits and its gradient
  add_rms_norm, rms_norm_backward     root-mean-square norm of x + residual, and its gradients
  gated_ff, gated_ff_backward         y = (act(x Wg^T) * (x Wu^T)) Wd^T (+ residual), and its gradients
  q8_matmul                           product of 8-bit codes with scales per row and output, optionally gated
  add_rms_norm_q8, quantize_rows      the norm, or plain rows, as 8-bit codes with a scale per row
  embed, embed_backward               rows of a table by index (categorical columns, tokens), and the table's gradient
  add_layer_norm, layer_norm_backward the norm with a mean and a bias, and its gradients
  dropout                             dropout whose mask is a function of (seed, step, site) and is never stored
  quantize_blocks, quantize_tiles     rows and weights as 8-bit floating point codes with a scale per block of 128
  f8_matmul                           product of those codes, optionally gated

Matrices are 2-D device tensors in bfloat16 or float32 whose rows are contiguous (any row stride and alignment).
Every call runs HIP kernels on the current stream of the tensors' device; ``PackError`` says what an argument
breaks.  Nothing is recorded for autograd: gradients come from the backward calls, and under grad mode a tensor that
requires a gradient is refused (``torch.no_grad()``, or the inside of an ``autograd.Function``, takes it).  Formulas
and rules for empty, masked and non-finite rows are in ``include/tabpack.h``.
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


# The current device's number without torch's check that the GPU is initialised (a device tensor is in hand).
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _fail(msg):
    raise PackError(msg)


@functools.lru_cache(maxsize=None)
def _function(fn):
    return getattr(tabpack.load_library(), fn)


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
    call = _function(fn)
    if dev == _current_device():
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


def _empty_as(x):
    """A dense tensor of a matrix's shape and type (the shorter way where the matrix is dense itself)."""
    return torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)


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


# ------------------------------------------------------------------ layer norm
def add_layer_norm(x, weight, bias=None, residual=None, eps=1e-5):
    """(y, v, mean, rstd): v = x + residual (x itself without one), mean and rstd = (mean (v - mean)^2 + eps)^(-1/2) per
    row, y = (v - mean) rstd weight + bias.  x, residual [rows, cols], weight and bias fp32 [cols]; y and v in x's type,
    mean and rstd fp32 [rows]."""
    xp, ldx, rp, ldr, wp, prec, rows, cols = _norm_inputs(x, weight, residual)
    bp = None if bias is None else _vector(bias, "bias", cols)
    v = x if residual is None else _empty_as(x)
    y, mean = _empty_as(x), _empty(x, rows, dtype=torch.float32)
    rstd = torch.empty_like(mean)
    _call("pack_add_layer_norm", x, (weight, bias, residual), xp, ldx, rp, ldr, wp, bp, prec, rows, cols, float(eps),
          None if residual is None else v.data_ptr(), cols, y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr())
    return y, v, mean, rstd


def layer_norm_backward(dy, v, weight, mean, rstd, dv=None):
    """(dx, dweight, dbias) of add_layer_norm: dx is the gradient of x and of the residual, dv the gradient that reaches
    the sum v on its other path (None: none).  dx in v's type, dweight and dbias fp32."""
    prec = _prec(v, "v")
    vp, ldv = _matrix(v, "v")
    yp, ldy = _matrix(dy, "dy", v.dtype, v.shape)
    rows, cols = v.shape
    dp, ldd = (None, 0) if dv is None else _matrix(dv, "dv", v.dtype, v.shape)
    wp, mp, rp = _vector(weight, "weight", cols), _vector(mean, "mean", rows), _vector(rstd, "rstd", rows)
    dx, dw = _empty_as(v), torch.empty_like(weight)
    db = torch.empty_like(weight)
    work = _empty(v, _bytes("pack_layer_norm_backward_workspace_size", rows, cols), dtype=torch.uint8)
    _call("pack_layer_norm_backward", v, (dy, weight, mean, rstd, dv), yp, ldy, vp, ldv, wp, mp, rp, dp, ldd, prec,
          rows, cols, dx.data_ptr(), cols, dw.data_ptr(), db.data_ptr(), work.data_ptr(), work.numel())
    return dx, dw, db


# --------------------------------------------------------------------- dropout
def dropout(x, p, seed, step, site=0, residual=None):
    """y = (residual +) x / (1 - p) where an element is kept, residual (or 0) elsewhere.  The mask follows from (seed,
    step, site, row, column) alone, so nothing of it is kept: x's gradient is ``dropout(dy, p, seed, step, site)``.
    x, residual [rows, cols]; p in [0, 1], taken by draws of 16 bits (the share kept is 1 - p rounded up to a multiple of
    2^-16; a p so near to 1 that this is past it by more than one part in 256 is refused); seed below 2^64; step (taken mod 2^32) a number, or a device tensor of one
    int64, which the kernel reads when it runs: a captured graph then draws new masks at each replay; site below 2^32
    tells the dropouts of one network apart."""
    prec = _prec(x, "x")
    xp, ldx = _matrix(x, "x")
    rows, cols = x.shape
    rp, ldr = (None, 0) if residual is None else _matrix(residual, "residual", x.dtype, x.shape)
    if isinstance(step, torch.Tensor):
        at, number = _vector(step.reshape(-1) if step.dim() == 0 else step, "step", 1, torch.int64), 0
    else:
        at, number = None, int(step) & 0xFFFFFFFFFFFFFFFF
    if not 0 <= seed < 1 << 64:
        _fail("seed must lie in [0, 2^64)")
    if not 0 <= site < 1 << 32:
        _fail("site must lie in [0, 2^32)")
    y = _empty_as(x)
    _call("pack_dropout", x, (residual, step if at else None), xp, ldx, rp, ldr, prec, rows, cols, float(p), int(seed),
          number, at, int(site), y.data_ptr(), cols)
    return y


# ------------------------------------------------------------------ embeddings
def _indices(idx):
    if not (isinstance(idx, torch.Tensor) and idx.is_cuda and idx.dtype in (torch.int32, torch.int64) and idx.dim() == 1
            and idx.is_contiguous()):
        _fail("idx must be a contiguous 1-D device tensor of int32 or int64")
    return idx.data_ptr(), int(idx.dtype == torch.int64), idx.shape[0]


def embed(idx, table, scale=1.0):
    """Rows of a table times a scale: table[idx] * scale, [tokens, cols] in the table's type.  idx [tokens] int32 or
    int64; a negative index gives a row of zeros, one past the table a row of NaN."""
    prec = _prec(table, "table")
    tp, ldt = _matrix(table, "table")
    rows, cols = table.shape
    ip, wide, tokens = _indices(idx)
    y = _empty(table, tokens, cols)
    _call("pack_embed", table, (idx,), ip, wide, tp, ldt, prec, tokens, rows, cols, float(scale), y.data_ptr(), cols)
    return y


def embed_backward(dy, idx, rows, scale=1.0):
    """The gradient of embed's table of ``rows`` rows from dy [tokens, cols], in dy's type: sums in fp32 and a fixed
    order, rounded once.  Indices that are negative or past the table add to no row."""
    prec = _prec(dy, "dy")
    dp, ldd = _matrix(dy, "dy")
    ip, wide, tokens = _indices(idx)
    if dy.shape[0] != tokens:
        _fail(f"dy must have {tokens} rows, not {dy.shape[0]}")
    cols = dy.shape[1]
    if not 1 <= rows < 1 << 31:
        _fail(f"rows={rows} must lie in [1, 2^31)")
    work = _work(dy, "pack_embed_backward_workspace_size", prec, tokens, rows, cols)
    dtable = _empty(dy, rows, cols)
    _call("pack_embed_backward", dy, (idx,), dp, ldd, ip, wide, prec, tokens, rows, cols, float(scale),
          dtable.data_ptr(), None if work is None else work.data_ptr(), 0 if work is None else work.numel())
    return dtable


# ------------------------------------------------------- 8-bit floating point
_E4M3 = torch.float8_e4m3fn
_BLOCK = 128  # PACK_F8_BLOCK


def quantize_blocks(x):
    """(q, scale): rows as e4m3 codes (float8_e4m3fn [rows, cols]) with a scale for each 128 columns of a row (fp32
    [ceil(cols / 128), rows], the order in which f8_matmul reads them)."""
    prec = _prec(x, "x")
    xp, ldx = _matrix(x, "x")
    rows, cols = x.shape
    q, scale = _empty(x, rows, cols, dtype=_E4M3), _empty(x, -(-cols // _BLOCK), rows, dtype=torch.float32)
    _call("pack_quantize_blocks", x, (), xp, ldx, prec, rows, cols, q.data_ptr(), cols, scale.data_ptr())
    return q, scale


def quantize_tiles(w, gated=False):
    """(q, scale): a weight [outputs, depth] as e4m3 codes with a scale for each 128 x 128 of it (fp32 [ceil(outputs /
    128), ceil(depth / 128)]).  gated: w holds gate rows and as many up rows, whose tiles begin anew and whose scales
    follow."""
    prec = _prec(w, "w")
    wp, ldw = _matrix(w, "w")
    rows, cols = w.shape
    parts = 2 if gated else 1
    if rows % parts:
        _fail("a gated w holds as many gate rows as up rows")
    q = _empty(w, rows, cols, dtype=_E4M3)
    scale = _empty(w, parts * -(-rows // parts // _BLOCK), -(-cols // _BLOCK), dtype=torch.float32)
    _call("pack_quantize_tiles", w, (), wp, ldw, prec, rows // parts, parts, cols, q.data_ptr(), cols, scale.data_ptr())
    return q, scale


def f8_matmul(q, scale, w, w_scale, bias=None, gate=None, dtype=torch.bfloat16):
    """x w^T (+ bias) of e4m3 codes q [rows, depth] and w [outputs, depth] with the scales of quantize_blocks and
    quantize_tiles, sums in fp32; [rows, outputs] in ``dtype``.  gate: an activation name; w, w_scale and bias then hold
    the gate rows and the up rows (``quantize_tiles(w, gated=True)``), and the result is act(gate) * up.  Results in
    float32 are summed from exact products, at half the rate; those in bfloat16 by the instructions for 8-bit codes,
    which cut off what lies 13 bits below the largest of 8 products (include/tabpack.h)."""
    qp, ldq = _matrix(q, "q", _E4M3)
    rows, depth = q.shape
    wp, ldw = _matrix(w, "w", _E4M3)
    n = w.shape[0]
    if w.shape[1] != depth:
        _fail(f"w must have {depth} columns, not {w.shape[1]}")
    code = -1 if gate is None else _act(gate)
    if gate is not None and n % 2:
        _fail("a gated w holds as many gate rows as up rows")
    if dtype not in _PREC:
        _fail("dtype must be bfloat16 or float32")
    outputs, blocks = n if gate is None else n // 2, -(-depth // _BLOCK)
    sp, _ = _matrix(scale, "scale", torch.float32, (blocks, rows))
    tiles = -(-outputs // _BLOCK) * (1 if gate is None else 2)
    wsp, _ = _matrix(w_scale, "w_scale", torch.float32, (tiles, blocks))
    if not (scale.is_contiguous() and w_scale.is_contiguous()):
        _fail("scale and w_scale must be contiguous")
    bp = None if bias is None else _vector(bias, "bias", n)
    out = _empty(q, rows, outputs, dtype=dtype)
    work = _work(q, "pack_f8_matmul_workspace_size", rows, outputs, depth, code)
    _call("pack_f8_matmul", q, (scale, w, w_scale, bias), qp, ldq, sp, wp, ldw, wsp, bp, code, _PREC[dtype], rows,
          outputs, depth, out.data_ptr(), outputs, None if work is None else work.data_ptr(),
          0 if work is None else work.numel())
    return out
