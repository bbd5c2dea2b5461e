"""ctypes binding of the operators that produce the gradients the step takes
(the C ABI in ``include/lionmuon_grad.h``, same library as ``lionmuon.py``).

* products grouped by expert: ``lionmuon_grouped_product`` and its gradients
  ``lionmuon_grouped_input_grad`` and ``lionmuon_grouped_weight_grad`` (fp32, the
  type that the step reads);
* 8-bit activation checkpoints: ``lionmuon_checkpoint``,
  ``lionmuon_checkpoint_restore``, and the operators that read them;
* activation functions: ``lionmuon_activation``, ``lionmuon_activation_grad``;
* root-mean-square norm: ``lionmuon_rmsnorm``, ``lionmuon_rmsnorm_grad``.

Argument marshalling only, as in ``lionmuon.py``: matrices are 2-D GPU tensors
whose rows are contiguous (they may lie apart), calls are asynchronous on
``stream`` (default: the current stream of the tensors' device), outputs that
are not passed in are allocated by torch. Autograd records none of it; tensors that
are passed in and written count as changed in place, so that a backward pass which
needs what they held before fails. There is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from .lionmuon import LM_ERR_INVALID_ARGUMENT, LM_OK, LionMuonError, _check, library

CHECKPOINT_BLOCK = 128               # LM_CHECKPOINT_BLOCK
RMSNORM_MAX_COLS = 16384             # LM_RMSNORM_MAX_COLS
ACTIVATIONS = {"gelu": 0, "swiglu": 1}

GRAD_EXPORTED = ("lionmuon_checkpoint", "lionmuon_checkpoint_restore", "lionmuon_activation",
                 "lionmuon_activation_grad", "lionmuon_rmsnorm", "lionmuon_rmsnorm_grad",
                 "lionmuon_rmsnorm_workspace_bytes", "lionmuon_grouped_product",
                 "lionmuon_grouped_input_grad", "lionmuon_grouped_weight_grad",
                 "lionmuon_grouped_workspace_bytes")

_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class lm_matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_uint32)]


class lm_stack(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("count", ctypes.c_int64), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("stride", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_uint32)]


class lm_checkpoint(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld_codes", ctypes.c_int64),
                ("ld_scales", ctypes.c_int64)]


_typed = None


def _lib():
    global _typed
    if _typed is None:
        lib = library()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        m, s, c = (ctypes.POINTER(t) for t in (lm_matrix, lm_stack, lm_checkpoint))
        for name, args in (
                ("lionmuon_checkpoint", [m, c, vp]),
                ("lionmuon_checkpoint_restore", [c, m, vp]),
                ("lionmuon_activation", [m, i32, m, c, vp]),
                ("lionmuon_activation_grad", [m, m, c, i32, m, m, vp]),
                ("lionmuon_rmsnorm", [m, m, vp, ctypes.c_double, m, m, vp, c, vp]),
                ("lionmuon_rmsnorm_grad", [m, m, c, vp, vp, m, m, vp, i32, vp, sz, vp]),
                ("lionmuon_rmsnorm_workspace_bytes", [i64, i64, ctypes.POINTER(sz)]),
                ("lionmuon_grouped_product", [m, s, vp, m, vp]),
                ("lionmuon_grouped_input_grad", [m, s, vp, m, vp]),
                ("lionmuon_grouped_weight_grad", [m, m, c, vp, s, i32, vp, sz, vp]),
                ("lionmuon_grouped_workspace_bytes", [i64, i64, i64, i64, ctypes.POINTER(sz)])):
            f = getattr(lib, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        _typed = lib
    return _typed


def _invalid(message):
    raise LionMuonError(LM_ERR_INVALID_ARGUMENT, message)


class Checkpoint:
    """8-bit checkpoint of a (rows, cols) tensor: e4m3 ``codes`` (uint8, rows
    16-byte aligned and a multiple of 16 bytes apart) and ``scales`` (uint8, one
    byte e + 127 for each 128 columns of a row); a code stands for its
    e4m3 value times 2^e. Each row of codes reaches to a multiple of 16 bytes (the
    operators write 0 behind the last code): ``codes`` are the first columns of a
    tensor with such rows."""

    __slots__ = ("shape", "device", "_buffer", "_place", "_codes", "_scales", "_layout")

    def __init__(self, codes, scales):
        if not isinstance(codes, torch.Tensor) or not isinstance(scales, torch.Tensor):
            raise TypeError("codes and scales must be torch.Tensors")
        self._buffer = self.shape = self.device = None
        self._codes = codes
        self._scales = scales
        self._described()

    @classmethod
    def empty(cls, rows, cols, device="cuda"):
        """An uninitialised checkpoint (filled by the operators that write one):
        its codes and scales lie in one allocation."""
        ld, blocks = -(-cols // 16) * 16, -(-cols // CHECKPOINT_BLOCK)
        ld_scales = -(-blocks // 4) * 4
        self = cls.__new__(cls)
        self._buffer = buffer = torch.empty(rows * (ld + ld_scales), dtype=torch.uint8, device=device)
        self.shape = torch.Size((rows, cols))
        self.device = buffer.device
        base = buffer.data_ptr()
        self._place = lm_checkpoint(base, base + rows * ld if base else 0, rows, cols, ld,
                                    ld_scales)
        return self

    @property
    def _desc(self):
        """The descriptor of a call: of the memory that the tensors have now."""
        if self._buffer is None:
            c, s = self._codes, self._scales
            if (c.data_ptr(), s.data_ptr(), c.shape, c.stride(), s.stride()) != self._layout:
                self._described()          # (all that the descriptor is made of)
            return self._place
        d = self._place
        base = self._buffer.data_ptr()
        if base != d.codes:
            d = self._place = lm_checkpoint(base, base + d.rows * d.ld_codes if base else 0, d.rows,
                                            d.cols, d.ld_codes, d.ld_scales)
        return d

    def _written(self):
        for t in (self._codes, self._scales) if self._buffer is None else (self._buffer,):
            _written(t)

    def _described(self):
        """Checks the tensors and describes them as they are now."""
        codes, scales = self._codes, self._scales
        for t in (codes, scales):
            if t.dtype != torch.uint8 or t.dim() != 2:
                _invalid(f"{'codes' if t is codes else 'scales'} must be a 2-D uint8 tensor")
        shape, device = codes.shape, codes.device
        if self.shape is None:
            self.shape, self.device = shape, device
        elif shape != self.shape or device != self.device:
            _invalid("codes have another shape or device than the checkpoint was made with")
        rows, cols = shape
        blocks = -(-cols // CHECKPOINT_BLOCK)
        if scales.shape != (rows, blocks):
            _invalid("scales must hold one byte for each 128 columns of a row")
        if device != scales.device:
            _invalid("codes and scales must be on one device")
        strides, strides_scales = codes.stride(), scales.stride()
        ld, step = strides
        ld_scales, step_scales = strides_scales
        if (cols > 1 and step != 1) or (blocks > 1 and step_scales != 1):
            _invalid("the rows of codes and scales must be contiguous")
        # a row's codes are written to the next multiple of 16: bytes of that row
        whole = -(-cols // 16) * 16
        if whole > cols and rows and (
                ld < whole or (rows - 1) * ld + whole > codes.untyped_storage().nbytes() - codes.storage_offset()):
            _invalid("the rows of codes must reach to a multiple of 16 bytes, the last one too")
        if rows > 1 and ld_scales % 4 == 0 and rows * ld_scales > \
                scales.untyped_storage().nbytes() - scales.storage_offset():
            _invalid("the last row of scales must be as long as the others")
        p, q = codes.data_ptr(), scales.data_ptr()
        self._place = lm_checkpoint(p, q, rows, cols, ld if rows > 1 else whole,
                                    ld_scales if rows > 1 else blocks)
        self._layout = (p, q, shape, strides, strides_scales)

    @property
    def codes(self):
        if self._buffer is None:
            return self._codes
        d = self._place
        return self._buffer[:d.rows * d.ld_codes].view(d.rows, d.ld_codes)[:, :d.cols]

    @property
    def scales(self):
        if self._buffer is None:
            return self._scales
        d = self._place
        return self._buffer[d.rows * d.ld_codes:].view(d.rows, d.ld_scales)[
            :, :-(-d.cols // CHECKPOINT_BLOCK)]


# -- marshalling -------------------------------------------------------------
def _device_of(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    device = t.device
    if device.type != "cuda":
        _invalid(f"{name} must be a GPU tensor")
    return device


def _check_place(t, name, device):
    if _device_of(t, name) != device:
        _invalid(f"{name} is on {t.device}, the other tensors are on {device}")


def _matrix(t, name, device):
    if not isinstance(t, torch.Tensor) or t.device != device:
        _check_place(t, name, device)
    code = _DTYPES.get(t.dtype)
    if code is None:
        _invalid(f"{name} must be float32, bfloat16 or float16")
    if t.dim() != 2:
        _invalid(f"{name} must be 2-D")
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        _invalid(f"the rows of {name} must be contiguous")
    return lm_matrix(t.data_ptr(), rows, cols, ld if rows > 1 else cols, code, 0)


def _new(rows, cols, like, code):
    """A new contiguous matrix of like's type and its descriptor."""
    t = torch.empty_like(like) if like.shape == (rows, cols) and like.is_contiguous() else \
        like.new_empty((rows, cols))
    return t, lm_matrix(t.data_ptr(), rows, cols, cols, code, 0)


def _stack(t, name, device):
    if not isinstance(t, torch.Tensor) or t.device != device:
        _check_place(t, name, device)
    code = _DTYPES.get(t.dtype)
    if code is None:
        _invalid(f"{name} must be float32, bfloat16 or float16")
    if t.dim() != 3:
        _invalid(f"{name} must be 3-D (experts, n, k)")
    count, rows, cols = t.shape
    stride, ld, step = t.stride()
    if step != 1 and cols > 1:
        _invalid(f"the rows of {name} must be contiguous")
    if rows <= 1:
        ld = cols
    return lm_stack(t.data_ptr(), count, rows, cols, ld, stride if count > 1 else rows * ld,
                    code, 0)


def _codes(c, name, device):
    if not isinstance(c, Checkpoint):
        raise TypeError(f"{name} must be a Checkpoint")
    if c.device != device:
        _invalid(f"{name} is on {c.device}, the other tensors are on {device}")
    return c._desc


def _wanted(checkpoint, rows, cols, device):
    """The Checkpoint to write and its descriptor: None, a new one, or the one passed in."""
    if checkpoint is False or checkpoint is None:
        return None, None
    if isinstance(checkpoint, Checkpoint):
        return checkpoint, _codes(checkpoint, "checkpoint", device)
    new = Checkpoint.empty(rows, cols, device)
    return new, new._place


def _vector(t, n, name, device):
    if not isinstance(t, torch.Tensor) or t.device != device:
        _check_place(t, name, device)
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        _invalid(f"{name} must be a contiguous float32 tensor of {n} values")
    return t.data_ptr()


def _offsets(t, experts, device):
    if not isinstance(t, torch.Tensor) or t.device != device:
        _check_place(t, "offsets", device)
    if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] != experts + 1 or \
            not t.is_contiguous():
        _invalid(f"offsets must be a contiguous int32 tensor of {experts + 1} values")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _here(device, stream):
    """Handle of the current stream if that is where the call goes, else None."""
    if stream is None and torch.cuda.current_device() == device.index:
        return _raw_stream(device.index)
    return None


@contextlib.contextmanager
def _switched(device, stream):
    """Makes the tensors' device and the call's stream current, so that what torch
    allocates for the call belongs to that stream."""
    with torch.cuda.device(device):
        if stream is None:
            yield
            return
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), device=device)
        elif stream.device != device:
            _invalid(f"stream is on {stream.device}, the tensors are on {device}")
        with torch.cuda.stream(stream):
            yield


def _done(status, what):
    if status != LM_OK:
        _check(status, what)


_written = torch.autograd.graph.increment_version      # of a tensor that was passed in


# -- checkpoints -------------------------------------------------------------
def lionmuon_checkpoint(x, out: Checkpoint | None = None, stream=None) -> Checkpoint:
    """8-bit checkpoint of a 2-D float32, bfloat16 or float16 tensor."""
    device = _device_of(x, "x")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_checkpoint(x, out)
    m = _matrix(x, "x", device)
    if out is None:
        kept = Checkpoint.empty(m.rows, m.cols, device)
        _done(_lib().lionmuon_checkpoint(m, kept._place, handle), "lionmuon_checkpoint")
        return kept
    _done(_lib().lionmuon_checkpoint(m, _codes(out, "out", device), handle), "lionmuon_checkpoint")
    out._written()
    return out


def lionmuon_checkpoint_restore(checkpoint: Checkpoint, dtype=torch.bfloat16, out=None,
                                stream=None):
    """The values of a checkpoint, in ``dtype`` (exact in float32 and bfloat16)."""
    if not isinstance(checkpoint, Checkpoint):
        raise TypeError("checkpoint must be a Checkpoint")
    device = checkpoint.device
    if device.type != "cuda":
        _invalid("checkpoint must be on a GPU")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_checkpoint_restore(checkpoint, dtype, out)
    x = torch.empty(checkpoint.shape, dtype=dtype, device=device) if out is None else out
    _done(_lib().lionmuon_checkpoint_restore(checkpoint._desc, _matrix(x, "out", device), handle),
          "lionmuon_checkpoint_restore")
    if out is not None:
        _written(out)
    return x


# -- activation functions ----------------------------------------------------
def _kind(kind):
    code = ACTIVATIONS.get(kind)
    if code is None:
        raise ValueError(f"unknown activation {kind!r}: one of {sorted(ACTIVATIONS)}")
    return code


def lionmuon_activation(a, kind, out=None, checkpoint=False, stream=None):
    """h = act(a): ``"gelu"`` (tanh form), or ``"swiglu"`` of a = [g | u].
    Returns (h, kept): kept is the checkpoint of a, written in the same pass, if
    ``checkpoint`` is true (or the Checkpoint to write), else None."""
    code = _kind(kind)
    device = _device_of(a, "a")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_activation(a, kind, out, checkpoint)
    m = _matrix(a, "a", device)
    rows, cols = m.rows, m.cols
    if code == 1 and cols % 2:
        _invalid("a must have an even number of columns")
    if out is None:
        h, mh = _new(rows, cols // (1 + code), a, m.dtype)
    else:
        h, mh = out, _matrix(out, "out", device)
    kept, mk = _wanted(checkpoint, rows, cols, device)
    _done(_lib().lionmuon_activation(m, code, mh, mk, handle), "lionmuon_activation")
    if out is not None:
        _written(out)
    if kept is checkpoint and kept is not None:
        kept._written()
    return h, kept


def lionmuon_activation_grad(dh, a, kind, out=None, recompute=False, stream=None):
    """da = dh * act'(a); ``a`` is the activation's input or its Checkpoint.
    Returns (da, h): h = act(a) again, from the same values, if ``recompute`` is
    true (or the tensor to write), else None."""
    code = _kind(kind)
    device = _device_of(dh, "dh")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_activation_grad(dh, a, kind, out, recompute)
    m = _matrix(dh, "dh", device)
    rows, cols = m.rows, m.cols
    ma = mk = None
    if isinstance(a, Checkpoint):
        mk = _codes(a, "a", device)
    else:
        ma = _matrix(a, "a", device)
    if out is None:
        da, mda = _new(rows, cols * (1 + code), dh, m.dtype)
    else:
        da, mda = out, _matrix(out, "out", device)
    if isinstance(recompute, torch.Tensor):
        h, mh = recompute, _matrix(recompute, "recompute", device)
    elif recompute:
        h, mh = _new(rows, cols, dh, m.dtype)
    else:
        h = mh = None
    _done(_lib().lionmuon_activation_grad(m, ma, mk, code, mda, mh, handle),
          "lionmuon_activation_grad")
    if out is not None:
        _written(out)
    if h is recompute and h is not None:
        _written(h)
    return da, h


# -- root-mean-square norm ---------------------------------------------------
def lionmuon_rmsnorm(x, weight, residual=None, eps=1e-5, out=None, sum_out=None,
                     checkpoint=False, stream=None):
    """Norm of s = x + residual (rounded to x's type; s = x without a residual):
    y = s * rstd * weight, rstd = 1 / sqrt(mean(s^2) + eps). ``weight``: float32.
    Returns (y, s, rstd, kept): y is None if ``out`` is False; s is x itself
    without a residual, else a new tensor or ``sum_out`` (which may be
    ``residual``); kept is the 8-bit checkpoint of y if ``checkpoint`` is true
    (or the Checkpoint to write), else None."""
    device = _device_of(x, "x")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_rmsnorm(x, weight, residual, eps, out, sum_out, checkpoint)
    m = _matrix(x, "x", device)
    rows, cols = m.rows, m.cols
    w = _vector(weight, cols, "weight", device)
    s, mr, ms = x, None, None
    if residual is not None:
        mr = _matrix(residual, "residual", device)
        if sum_out is None:
            s, ms = _new(rows, cols, x, m.dtype)
        else:
            s, ms = sum_out, _matrix(sum_out, "sum_out", device)
    elif sum_out is not None:
        _invalid("sum_out needs a residual")
    if out is None:
        y, my = _new(rows, cols, x, m.dtype)
    elif out is False:
        y = my = None
    else:
        y, my = out, _matrix(out, "out", device)
    rstd = weight.new_empty(rows)
    kept, mk = _wanted(checkpoint, rows, cols, device)
    _done(_lib().lionmuon_rmsnorm(m, mr, w, eps, my, ms, rstd.data_ptr(), mk, handle),
          "lionmuon_rmsnorm")
    if out is not None and y is not None:
        _written(y)
    if sum_out is not None:
        _written(sum_out)
    if kept is checkpoint and kept is not None:
        kept._written()
    return y, s, rstd, kept


def lionmuon_rmsnorm_grad(dy, s, weight, rstd, residual_grad=None, out=None, weight_grad=None,
                          accumulate=False, stream=None):
    """Gradients (dx, dweight) of lionmuon_rmsnorm. ``s``: the normed stream or its
    Checkpoint; ``residual_grad``: gradient that reaches s past the norm, added to
    dx (``out`` may be that tensor). dx is the gradient of x and of the residual;
    dweight is float32, written to ``weight_grad`` (added to it with
    ``accumulate``). ``weight_grad=False`` or ``out=False`` leaves one out (None)."""
    device = _device_of(dy, "dy")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_rmsnorm_grad(dy, s, weight, rstd, residual_grad, out, weight_grad,
                                         accumulate)
    m = _matrix(dy, "dy", device)
    rows, cols = m.rows, m.cols
    ms = mk = None
    if isinstance(s, Checkpoint):
        mk = _codes(s, "s", device)
    else:
        ms = _matrix(s, "s", device)
    mr = None if residual_grad is None else _matrix(residual_grad, "residual_grad", device)
    w = _vector(weight, cols, "weight", device)
    r = _vector(rstd, rows, "rstd", device)
    if accumulate and not isinstance(weight_grad, torch.Tensor):
        _invalid("accumulate needs weight_grad")
    if out is None:
        dx, mdx = _new(rows, cols, dy, m.dtype)
    elif out is False:
        dx = mdx = None
    else:
        dx, mdx = out, _matrix(out, "out", device)
    dw = pw = ws = None
    nbytes = 0
    if weight_grad is not False:
        if weight_grad is None:
            dw = torch.empty_like(weight)
            pw = dw.data_ptr()
        else:
            dw, pw = weight_grad, _vector(weight_grad, cols, "weight_grad", device)
        nbytes = lionmuon_rmsnorm_workspace_bytes(rows, cols)
        if nbytes:
            ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    _done(_lib().lionmuon_rmsnorm_grad(m, ms, mk, w, r, mr, mdx, pw, 1 if accumulate else 0,
                                       None if ws is None else ws.data_ptr(), nbytes, handle),
          "lionmuon_rmsnorm_grad")
    if out is not None and dx is not None:
        _written(dx)
    if weight_grad is not None and dw is not None:
        _written(dw)
    return dx, dw


def lionmuon_rmsnorm_workspace_bytes(rows, cols) -> int:
    out = ctypes.c_size_t(0)
    _done(_lib().lionmuon_rmsnorm_workspace_bytes(rows, cols, out),
          "lionmuon_rmsnorm_workspace_bytes")
    return out.value


# -- products grouped by expert ----------------------------------------------
def lionmuon_grouped_product(x, w, offsets, out=None, stream=None):
    """Y[r] = X[r] W_e^T for the rows offsets[e] <= r < offsets[e + 1] of each expert
    e. x: (T, k), w: (experts, n, k), both bfloat16 or float16; offsets: int32 GPU
    tensor of experts + 1 values. Rows of no expert keep what ``out`` holds
    (a new ``out`` is not initialised there)."""
    device = _device_of(x, "x")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_grouped_product(x, w, offsets, out)
    m = _matrix(x, "x", device)
    mw = _stack(w, "w", device)
    at = _offsets(offsets, mw.count, device)
    if out is None:
        y, mo = _new(m.rows, mw.rows, x, m.dtype)
    else:
        y, mo = out, _matrix(out, "out", device)
    _done(_lib().lionmuon_grouped_product(m, mw, at, mo, handle), "lionmuon_grouped_product")
    if out is not None:
        _written(out)
    return y


def lionmuon_grouped_input_grad(dy, w, offsets, out=None, stream=None):
    """dX[r] = dY[r] W_e (see lionmuon_grouped_product). dy: (T, n)."""
    device = _device_of(dy, "dy")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_grouped_input_grad(dy, w, offsets, out)
    m = _matrix(dy, "dy", device)
    mw = _stack(w, "w", device)
    at = _offsets(offsets, mw.count, device)
    if out is None:
        dx, mo = _new(m.rows, mw.cols, dy, m.dtype)
    else:
        dx, mo = out, _matrix(out, "out", device)
    _done(_lib().lionmuon_grouped_input_grad(m, mw, at, mo, handle), "lionmuon_grouped_input_grad")
    if out is not None:
        _written(out)
    return dx


def lionmuon_grouped_weight_grad(dy, x, offsets, out=None, accumulate=False, stream=None):
    """dW_e = dY_e^T X_e, float32 (experts, n, k); added to ``out`` with
    ``accumulate``. ``x``: (T, k) tensor of dy's type or its Checkpoint (dy must then
    be bfloat16). ``out.unbind()`` are gradients as the step takes them."""
    device = _device_of(dy, "dy")
    handle = _here(device, stream)
    if handle is None:
        with _switched(device, stream):
            return lionmuon_grouped_weight_grad(dy, x, offsets, out, accumulate)
    m = _matrix(dy, "dy", device)
    mx = mk = None
    if isinstance(x, Checkpoint):
        mk = _codes(x, "x", device)
        cols = mk.cols
    else:
        mx = _matrix(x, "x", device)
        cols = mx.cols
    if out is None:
        if accumulate:
            _invalid("accumulate needs out")
        # (no value is one too few for no expert, which the workspace's size refuses)
        experts = max(offsets.numel() - 1, 0) if isinstance(offsets, torch.Tensor) else 0
        at = _offsets(offsets, experts, device)
        dw = torch.empty((experts, m.cols, cols), dtype=torch.float32, device=device)
        mo = lm_stack(dw.data_ptr(), experts, m.cols, cols, cols, m.cols * cols, 0, 0)
    else:
        dw, mo = out, _stack(out, "out", device)
        experts = mo.count
        at = _offsets(offsets, experts, device)
    nbytes = lionmuon_grouped_workspace_bytes(m.rows, experts, m.cols, cols)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    _done(_lib().lionmuon_grouped_weight_grad(m, mx, mk, at, mo, 1 if accumulate else 0,
                                              None if ws is None else ws.data_ptr(), nbytes,
                                              handle), "lionmuon_grouped_weight_grad")
    if out is not None:
        _written(out)
    return dw


def lionmuon_grouped_workspace_bytes(rows, experts, n, k) -> int:
    out = ctypes.c_size_t(0)
    _done(_lib().lionmuon_grouped_workspace_bytes(rows, experts, n, k, out),
          "lionmuon_grouped_workspace_bytes")
    return out.value
