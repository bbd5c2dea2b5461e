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
are not passed in are allocated by torch. Autograd sees none of it. There is
no fallback.
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
    e4m3 value times 2^e."""

    __slots__ = ("codes", "scales")

    def __init__(self, codes, scales):
        for t, name in ((codes, "codes"), (scales, "scales")):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch.Tensor")
            if t.dtype != torch.uint8 or t.dim() != 2:
                _invalid(f"{name} must be a 2-D uint8 tensor")
        if scales.shape != (codes.shape[0], -(-codes.shape[1] // CHECKPOINT_BLOCK)):
            _invalid("scales must hold one byte for each 128 columns of a row")
        if codes.device != scales.device:
            _invalid("codes and scales must be on one device")
        self.codes = codes
        self.scales = scales

    @classmethod
    def empty(cls, rows, cols, device=None):
        """An uninitialised checkpoint (filled by the operators that write one)."""
        codes = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=device or "cuda")
        scales = torch.empty(rows, -(-cols // CHECKPOINT_BLOCK), dtype=torch.uint8,
                             device=codes.device)
        return cls(codes[:, :cols], scales)

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device


# -- marshalling -------------------------------------------------------------
def _matrix(t, name, device=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        _invalid(f"{name} must be a GPU tensor")
    if device is not None and t.device != device:
        _invalid(f"{name} is on {t.device}, the other tensors are on {device}")
    if t.dim() != 2:
        _invalid(f"{name} must be 2-D")
    code = _DTYPES.get(t.dtype)
    if code is None:
        _invalid(f"{name} must be float32, bfloat16 or float16")
    rows, cols = t.shape
    ld, step = t.stride()
    if cols > 1 and step != 1:
        _invalid(f"the rows of {name} must be contiguous")
    return lm_matrix(t.data_ptr(), rows, cols, ld if rows > 1 else cols, code, 0)


def _stack(t, name, device):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda or t.device != device:
        _invalid(f"{name} must be on {device}")
    if t.dim() != 3:
        _invalid(f"{name} must be 3-D (experts, n, k)")
    code = _DTYPES.get(t.dtype)
    if code is None:
        _invalid(f"{name} must be float32, bfloat16 or float16")
    count, rows, cols = t.shape
    stride, ld, step = t.stride()
    if cols > 1 and step != 1:
        _invalid(f"the rows of {name} must be contiguous")
    ld = ld if rows > 1 else cols
    return lm_stack(t.data_ptr(), count, rows, cols, ld,
                    stride if count > 1 else rows * ld, code, 0)


def _codes(c, name, device):
    if not isinstance(c, Checkpoint):
        raise TypeError(f"{name} must be a Checkpoint")
    if not c.codes.is_cuda or c.codes.device != device:
        _invalid(f"{name} must be on {device}")
    rows, cols = c.codes.shape
    ld, step = c.codes.stride()
    ld_scales, step_scales = c.scales.stride()
    blocks = c.scales.shape[1]
    if (cols > 1 and step != 1) or (blocks > 1 and step_scales != 1):
        _invalid(f"the rows of {name} must be contiguous")
    return lm_checkpoint(c.codes.data_ptr(), c.scales.data_ptr(), rows, cols,
                         ld if rows > 1 else -(-cols // 16) * 16,
                         ld_scales if rows > 1 else blocks)


def _vector(t, n, name, device):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda or t.device != device:
        _invalid(f"{name} must be on {device}")
    if t.dtype != torch.float32 or t.shape != (n,) or not t.is_contiguous():
        _invalid(f"{name} must be a contiguous float32 tensor of {n} values")
    return t.data_ptr()


def _offsets(t, experts, device):
    if not isinstance(t, torch.Tensor):
        raise TypeError("offsets must be a torch.Tensor")
    if not t.is_cuda or t.device != device:
        _invalid(f"offsets must be on {device}")
    if t.dtype != torch.int32 or t.shape != (experts + 1,) or not t.is_contiguous():
        _invalid(f"offsets must be a contiguous int32 tensor of {experts + 1} values")
    return t.data_ptr()


def _ref(x):
    return None if x is None else ctypes.byref(x)


@contextlib.contextmanager
def _switched(device, stream):
    with torch.cuda.device(device):
        if stream is None:
            yield torch.cuda.current_stream().cuda_stream
            return
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), device=device)
        elif stream.device != device:
            _invalid(f"stream is on {stream.device}, the tensors are on {device}")
        # what torch allocates for the call belongs to the call's stream
        with torch.cuda.stream(stream):
            yield stream.cuda_stream


@contextlib.contextmanager
def _unswitched(handle):
    yield handle


def _stream(device, stream):
    """Context in which a call on `device` and `stream` allocates and launches."""
    if stream is None and torch.cuda.current_device() == device.index:
        return _unswitched(torch.cuda.current_stream().cuda_stream)
    return _switched(device, stream)


def _device_of(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        _invalid(f"{name} must be a GPU tensor")
    return t.device


def _done(status, what):
    if status != LM_OK:
        _check(status, what)


# -- checkpoints -------------------------------------------------------------
def lionmuon_checkpoint(x, out: Checkpoint | None = None, stream=None) -> Checkpoint:
    """8-bit checkpoint of a 2-D float32, bfloat16 or float16 tensor."""
    device = _device_of(x, "x")
    mx = _matrix(x, "x")
    with _stream(device, stream) as handle:
        if out is None:
            out = Checkpoint.empty(mx.rows, mx.cols, device)
        _done(_lib().lionmuon_checkpoint(mx, _codes(out, "out", device), handle),
              "lionmuon_checkpoint")
    return out


def lionmuon_checkpoint_restore(checkpoint: Checkpoint, dtype=torch.bfloat16, out=None,
                                stream=None):
    """The values of a checkpoint, in ``dtype`` (exact in float32 and bfloat16)."""
    if not isinstance(checkpoint, Checkpoint):
        raise TypeError("checkpoint must be a Checkpoint")
    device = _device_of(checkpoint.codes, "checkpoint")
    with _stream(device, stream) as handle:
        if out is None:
            out = torch.empty(checkpoint.shape, dtype=dtype, device=device)
        _done(_lib().lionmuon_checkpoint_restore(_codes(checkpoint, "checkpoint", device),
                                                 _matrix(out, "out", device), handle),
              "lionmuon_checkpoint_restore")
    return out


# -- activation functions ----------------------------------------------------
def _kind(kind):
    if kind not in ACTIVATIONS:
        raise ValueError(f"unknown activation {kind!r}: one of {sorted(ACTIVATIONS)}")
    return ACTIVATIONS[kind]


def lionmuon_activation(a, kind, out=None, checkpoint=False, stream=None):
    """h = act(a): ``"gelu"`` (tanh form), or ``"swiglu"`` of a = [g | u].
    Returns (h, kept): kept is the checkpoint of a, written in the same pass, if
    ``checkpoint`` is true (or the Checkpoint to write), else None."""
    code = _kind(kind)
    device = _device_of(a, "a")
    ma = _matrix(a, "a")
    if code == 1 and ma.cols % 2:
        _invalid("a must have an even number of columns")
    with _stream(device, stream) as handle:
        if out is None:
            out = torch.empty(ma.rows, ma.cols // (1 + code), dtype=a.dtype, device=device)
        kept = _wanted(checkpoint, ma.rows, ma.cols, device)
        mk = None if kept is None else _codes(kept, "checkpoint", device)
        _done(_lib().lionmuon_activation(ma, code, _matrix(out, "out", device), _ref(mk), handle),
              "lionmuon_activation")
    return out, kept


def _wanted(checkpoint, rows, cols, device):
    if isinstance(checkpoint, Checkpoint):
        return checkpoint
    return Checkpoint.empty(rows, cols, device) if checkpoint else None


def lionmuon_activation_grad(dh, a, kind, out=None, recompute=False, stream=None):
    """da = dh * act'(a); ``a`` is the activation's input or its Checkpoint.
    Returns (da, h): h = act(a) again, from the same values, if ``recompute`` is
    true (or the tensor to write), else None."""
    code = _kind(kind)
    device = _device_of(dh, "dh")
    md = _matrix(dh, "dh")
    kept = isinstance(a, Checkpoint)
    ma = None if kept else _matrix(a, "a", device)
    mk = _codes(a, "a", device) if kept else None
    with _stream(device, stream) as handle:
        if out is None:
            out = torch.empty(md.rows, md.cols * (1 + code), dtype=dh.dtype, device=device)
        h = recompute if isinstance(recompute, torch.Tensor) else \
            torch.empty(md.rows, md.cols, dtype=dh.dtype, device=device) if recompute else None
        mh = None if h is None else _matrix(h, "recompute", device)
        _done(_lib().lionmuon_activation_grad(md, _ref(ma), _ref(mk), code,
                                              _matrix(out, "out", device), _ref(mh), handle),
              "lionmuon_activation_grad")
    return out, h


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
    mx = _matrix(x, "x")
    mr = None if residual is None else _matrix(residual, "residual", device)
    if sum_out is not None and residual is None:
        _invalid("sum_out needs a residual")
    w = _vector(weight, mx.cols, "weight", device)
    with _stream(device, stream) as handle:
        y = None if out is False else torch.empty_like(x, memory_format=torch.contiguous_format) \
            if out is None else out
        my = None if y is None else _matrix(y, "out", device)
        s, ms = x, None
        if residual is not None:
            s = torch.empty_like(x, memory_format=torch.contiguous_format) if sum_out is None \
                else sum_out
            ms = _matrix(s, "sum_out", device)
        rstd = torch.empty(mx.rows, dtype=torch.float32, device=device)
        kept = _wanted(checkpoint, mx.rows, mx.cols, device)
        mk = None if kept is None else _codes(kept, "checkpoint", device)
        _done(_lib().lionmuon_rmsnorm(mx, _ref(mr), w, eps, _ref(my), _ref(ms), rstd.data_ptr(),
                                      _ref(mk), handle), "lionmuon_rmsnorm")
    return y, s, rstd, kept


def lionmuon_rmsnorm_grad(dy, s, weight, rstd, residual_grad=None, out=None, weight_grad=None,
                          accumulate=False, stream=None):
    """Gradients (dx, dweight) of lionmuon_rmsnorm. ``s``: the normed stream or its
    Checkpoint; ``residual_grad``: gradient that reaches s past the norm, added to
    dx (``out`` may be that tensor). dx is the gradient of x and of the residual;
    dweight is float32, written to ``weight_grad`` (added to it with
    ``accumulate``). ``weight_grad=False`` or ``out=False`` leaves one out (None)."""
    device = _device_of(dy, "dy")
    md = _matrix(dy, "dy")
    kept = isinstance(s, Checkpoint)
    ms = None if kept else _matrix(s, "s", device)
    mk = _codes(s, "s", device) if kept else None
    mr = None if residual_grad is None else _matrix(residual_grad, "residual_grad", device)
    w = _vector(weight, md.cols, "weight", device)
    r = _vector(rstd, md.rows, "rstd", device)
    lib = _lib()
    if accumulate and not isinstance(weight_grad, torch.Tensor):
        _invalid("accumulate needs weight_grad")
    with _stream(device, stream) as handle:
        dx = None if out is False else torch.empty_like(dy, memory_format=torch.contiguous_format) \
            if out is None else out
        mdx = None if dx is None else _matrix(dx, "out", device)
        dw, ws, nbytes = None, None, 0
        if weight_grad is not False:
            dw = torch.empty(md.cols, dtype=torch.float32, device=device) if weight_grad is None \
                else weight_grad
            nbytes = lionmuon_rmsnorm_workspace_bytes(md.rows, md.cols)
            if nbytes:
                ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        pw = None if dw is None else _vector(dw, md.cols, "weight_grad", device)
        _done(lib.lionmuon_rmsnorm_grad(md, _ref(ms), _ref(mk), w, r, _ref(mr), _ref(mdx), pw,
                                        1 if accumulate else 0,
                                        None if ws is None else ws.data_ptr(), nbytes, handle),
              "lionmuon_rmsnorm_grad")
    return dx, dw


def lionmuon_rmsnorm_workspace_bytes(rows, cols) -> int:
    out = ctypes.c_size_t(0)
    _done(_lib().lionmuon_rmsnorm_workspace_bytes(rows, cols, ctypes.byref(out)),
          "lionmuon_rmsnorm_workspace_bytes")
    return out.value


# -- products grouped by expert ----------------------------------------------
def lionmuon_grouped_product(x, w, offsets, out=None, stream=None):
    """Y[r] = X[r] W_e^T for the rows offsets[e] <= r < offsets[e + 1] of each expert
    e. x: (T, k), w: (experts, n, k), both bfloat16 or float16; offsets: int32 GPU
    tensor of experts + 1 values. Rows of no expert keep what ``out`` holds
    (a new ``out`` is not initialised there)."""
    device = _device_of(x, "x")
    mx = _matrix(x, "x")
    mw = _stack(w, "w", device)
    at = _offsets(offsets, mw.count, device)
    with _stream(device, stream) as handle:
        if out is None:
            out = torch.empty(mx.rows, mw.rows, dtype=x.dtype, device=device)
        _done(_lib().lionmuon_grouped_product(mx, mw, at, _matrix(out, "out", device), handle),
              "lionmuon_grouped_product")
    return out


def lionmuon_grouped_input_grad(dy, w, offsets, out=None, stream=None):
    """dX[r] = dY[r] W_e (see lionmuon_grouped_product). dy: (T, n)."""
    device = _device_of(dy, "dy")
    md = _matrix(dy, "dy")
    mw = _stack(w, "w", device)
    at = _offsets(offsets, mw.count, device)
    with _stream(device, stream) as handle:
        if out is None:
            out = torch.empty(md.rows, mw.cols, dtype=dy.dtype, device=device)
        _done(_lib().lionmuon_grouped_input_grad(md, mw, at, _matrix(out, "out", device), handle),
              "lionmuon_grouped_input_grad")
    return out


def lionmuon_grouped_weight_grad(dy, x, offsets, out=None, accumulate=False, stream=None):
    """dW_e = dY_e^T X_e, float32 (experts, n, k); added to ``out`` with
    ``accumulate``. ``x``: (T, k) tensor of dy's type or its Checkpoint (dy must then
    be bfloat16). ``out.unbind()`` are gradients as the step takes them."""
    device = _device_of(dy, "dy")
    md = _matrix(dy, "dy")
    kept = isinstance(x, Checkpoint)
    mx = None if kept else _matrix(x, "x", device)
    mk = _codes(x, "x", device) if kept else None
    cols = (mk or mx).cols
    if not isinstance(offsets, torch.Tensor):
        raise TypeError("offsets must be a torch.Tensor")
    if accumulate and out is None:
        _invalid("accumulate needs out")
    experts = offsets.numel() - 1 if out is None else out.shape[0]
    at = _offsets(offsets, experts, device)
    with _stream(device, stream) as handle:
        if out is None:
            out = torch.empty(experts, md.cols, cols, dtype=torch.float32, device=device)
        mo = _stack(out, "out", device)
        nbytes = lionmuon_grouped_workspace_bytes(md.rows, experts, md.cols, cols)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
        _done(_lib().lionmuon_grouped_weight_grad(md, _ref(mx), _ref(mk), at, mo,
                                                  1 if accumulate else 0,
                                                  None if ws is None else ws.data_ptr(), nbytes,
                                                  handle), "lionmuon_grouped_weight_grad")
    return out


def lionmuon_grouped_workspace_bytes(rows, experts, n, k) -> int:
    out = ctypes.c_size_t(0)
    _done(_lib().lionmuon_grouped_workspace_bytes(rows, experts, n, k, ctypes.byref(out)),
          "lionmuon_grouped_workspace_bytes")
    return out.value
