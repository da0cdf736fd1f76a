"""Python binding of the operators that a rematerialisation plan is run with (C ABI in
include/moccasin_training.h, in the same library as the evaluator).

Argument marshalling only, as in `moccasin`: tensors are checked and turned into descriptors (natively,
binding/training.cpp), results and workspaces are torch tensors, everything is asynchronous on `stream`
(default: torch's current stream) on the current device, where the tensors have to be.  Matrices are
two-dimensional CUDA tensors whose values of a row lie next to each other; rows may be any distance apart.  An `out` or `keep` that shares memory with an input is refused; it may be x of
moc_norm_forward, dy, x or residual of moc_norm_backward, residual of moc_linear_forward and pre of
moc_linear_backward_input themselves (same type and strides).  There is no CPU fallback: a missing library or GPU raises.

No call records a graph: results never require gradients, those of tensors that do included.  The gradients are calls of their
own (moc_*_backward*); inside torch's autograd they belong into the backward of a torch.autograd.Function.

A `Checkpoint` is an activation kept in 8 bits: a byte a value and a scale for 32 columns of a row.
"""
from __future__ import annotations

import collections
import ctypes

from . import moccasin as moc

MOC_TRAINING_VERSION = 2
MOC_F32, MOC_F16, MOC_BF16, MOC_E4M3, MOC_I8 = range(5)
FORMATS = {"e4m3": MOC_E4M3, "int8": MOC_I8}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
PRODUCTS = {"forward": 0, "backward_input": 1, "backward_weight": 2}
BLOCK = 32

EXPORTS = ("moc_checkpoint_write", "moc_checkpoint_read", "moc_norm_forward", "moc_norm_backward", "moc_norm_backward_work", "moc_linear_forward",
           "moc_linear_backward_input", "moc_linear_backward_weight", "moc_linear_work", "moc_linear_parts", "moc_training_version")


class Matrix(ctypes.Structure):
    """moc_matrix"""
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("stride", ctypes.c_int64), ("scale_stride", ctypes.c_int64),
                ("type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class Checkpoint:
    """An activation kept in 8 bits: `codes` uint8 [rows, cols], `scales` uint8 [rows, ceil(cols / 32)],
    `fmt` "e4m3" or "int8"."""

    __slots__ = ("codes", "scales", "fmt")

    def __init__(self, codes, scales, fmt):
        if fmt not in FORMATS:
            raise ValueError(f"checkpoint format {fmt!r}: expected one of {', '.join(FORMATS)}")
        self.codes, self.scales, self.fmt = codes, scales, fmt

    @property
    def shape(self):
        return self.codes.shape

    @property
    def nbytes(self):
        return self.codes.numel() + self.scales.numel()


_lib = None
_native = None


def lib():
    """The evaluator's library, with these operators in it."""
    global _lib
    if _lib is None:
        L = moc.lib()
        version = L.moc_training_version() if hasattr(L, "moc_training_version") else 0
        if version != MOC_TRAINING_VERSION:
            raise RuntimeError(f"{moc.LIB_PATH} has version {version} of the training operators, this binding needs {MOC_TRAINING_VERSION}; "
                               "run python -m paper_2304_14463_amd.build")
        I32, I64, VP, F32, M = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.POINTER(Matrix)
        for name, args in (("moc_checkpoint_write", [I64, I64, M, M, VP]),
                           ("moc_checkpoint_read", [I64, I64, M, I32, M, VP]),
                           ("moc_norm_forward", [I64, I64, M, VP, VP, I32, F32, M, M, VP, VP, VP]),
                           ("moc_norm_backward", [I64, I64, M, M, VP, I32, VP, VP, M, M, VP, VP, VP, I64, VP]),
                           ("moc_linear_forward", [I64, I64, I64, M, M, VP, I32, I32, M, M, M, VP, I64, VP]),
                           ("moc_linear_backward_input", [I64, I64, I64, M, M, I32, M, M, VP, I64, VP]),
                           ("moc_linear_backward_weight", [I64, I64, I64, M, M, M, VP, VP, I64, VP])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, ctypes.c_int
        for name, args in (("moc_norm_backward_work", [I64, I64]), ("moc_linear_work", [I64, I64, I64])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, I64
        L.moc_linear_parts.argtypes, L.moc_linear_parts.restype = [I32, I64, I64, I64, I32, I32, ctypes.POINTER(I64)], ctypes.c_int
        _lib = L
    return _lib


def _bound():
    """The native part of the binding (binding/training.cpp), loaded on first use: it needs torch."""
    global _native
    if _native is None:
        L = lib()
        moc._tc()
        try:
            from . import _training as native   # built with the library
        except ImportError as err:
            raise RuntimeError(f"{moc.LIB_PATH}: the binding's native part does not load ({err}); run python -m paper_2304_14463_amd.build") from err
        if getattr(native, "training_version", None) != MOC_TRAINING_VERSION:
            raise RuntimeError(f"{native.__file__}: version {getattr(native, 'training_version', None)} of the training operators, expected "
                               f"{MOC_TRAINING_VERSION}; run python -m paper_2304_14463_amd.build")
        native.bind(Checkpoint, _current_stream, {name: ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in EXPORTS})
        _native = native
    return _native


def _act(act):
    if act not in ACTS:
        raise ValueError(f"act {act!r}: expected one of {', '.join(ACTS)}")
    return ACTS[act]


def _current_stream(device):
    """Handle of the current stream.  Kernels run on the current device, as with moc_eval_batch's graph: tensors on another are
    refused."""
    torch = moc._tc()
    current = torch.cuda.current_device()
    if device != current:
        raise ValueError(f"tensors on cuda:{device}, the current device is cuda:{current}")
    return torch._C._cuda_getCurrentRawStream(current)


def _call(name, stream, *args):
    """(code, results..) of a native call; what it allocates belongs to `stream`, which is the current one meanwhile."""
    call = getattr(_native or _bound(), name)
    if stream is None:
        return call(*args)
    with moc._on(stream):
        return call(*args)


def empty_checkpoint(rows, cols, fmt, device):
    """Room for a checkpoint; its contents are undefined until a call has written it."""
    torch = moc._tc()
    return Checkpoint(torch.empty((rows, cols), dtype=torch.uint8, device=device), torch.empty((rows, -(-cols // BLOCK)), dtype=torch.uint8, device=device), fmt)


def moc_checkpoint_write(x, fmt="e4m3", out=None, stream=None):
    """Keep x [rows, cols] in 8 bits ("e4m3" or "int8").  Returns the Checkpoint (`out`, if given)."""
    code, out = _call("checkpoint_write", stream, x, fmt, out)
    moc._check(code, "moc_checkpoint_write")
    return out


def moc_checkpoint_read(kept, dtype, act="none", out=None, stream=None):
    """act(the values of a checkpoint), as a tensor of `dtype`."""
    code, out = _call("checkpoint_read", stream, kept, dtype, _act(act), out)
    moc._check(code, "moc_checkpoint_read")
    return out


def moc_norm_forward(x, gamma=None, beta=None, eps=1e-5, keep=None, dtype=None, out=None, stream=None):
    """Layer norm of the rows of x (a tensor or a Checkpoint).  Returns (y, mean, rstd, kept): y of
    `dtype` (default x's, float32 for a checkpoint), mean and rstd float32 [rows], and y in 8 bits if
    `keep` names a format or is a Checkpoint to write to, else None."""
    code, out, mean, rstd, kept = _call("norm_forward", stream, x, gamma, beta, eps, keep, dtype, out)
    moc._check(code, "moc_norm_forward")
    return out, mean, rstd, kept


def moc_norm_backward(dy, x, gamma, mean, rstd, residual=None, want_params=True, out=None, work=None, stream=None):
    """Layer norm's gradients from dy, x (a tensor or a Checkpoint) and the statistics of the forward
    pass.  Returns (dx of dy's type, dgamma, dbeta float32 or None); `residual` is added to dx."""
    code, out, dgamma, dbeta = _call("norm_backward", stream, dy, x, gamma, mean, rstd, residual, want_params, out, work)
    moc._check(code, "moc_norm_backward")
    return out, dgamma, dbeta


def moc_linear_forward(x, w, bias=None, act="none", residual=None, keep=None, dtype=None, out=None, work=None, stream=None):
    """act(x w^T + bias) + residual for x [rows, cin], w [cout, cin].  Returns (y of `dtype`, default
    x's; x w^T + bias in 8 bits if `keep` names a format or is a Checkpoint to write to, else None)."""
    code, out, kept = _call("linear_forward", stream, x, w, bias, _act(act), residual, keep, dtype, out, work)
    moc._check(code, "moc_linear_forward")
    return out, kept


def moc_linear_backward_input(dy, w, act="none", pre=None, dtype=None, out=None, work=None, stream=None):
    """(dy w) * act'(pre) for dy [rows, cout], w [cout, cin] and pre [rows, cin], a tensor or a
    Checkpoint of the activation's argument (act "none": no factor)."""
    code, out = _call("linear_backward_input", stream, dy, w, _act(act), pre, dtype, out, work)
    moc._check(code, "moc_linear_backward_input")
    return out


def moc_linear_backward_weight(dy, x, dtype=None, want_bias=True, out=None, work=None, stream=None):
    """(dw = dy^T x, db = the column sums of dy, float32 or None) for dy [rows, cout] and x [rows, cin],
    a tensor or a Checkpoint; dw [cout, cin] of `dtype`, default float32."""
    code, out, db = _call("linear_backward_weight", stream, dy, x, dtype, want_bias, out, work)
    moc._check(code, "moc_linear_backward_weight")
    return out, db


Parts = collections.namedtuple("Parts", "tile direct parts terms last")


def moc_linear_parts(product, rows, cin, cout, aligned=True, units=0):
    """How the product of moc_linear_`product` ("forward", "backward_input", "backward_weight") is cut up on a device of `units`
    compute units (0: the current one): rows and columns of a workgroup's tile, whether operands go straight into LDS, the
    parts of the sum, terms of a part and of the last one."""
    if product not in PRODUCTS:
        raise ValueError(f"product {product!r}: expected one of {', '.join(PRODUCTS)}")
    out = (ctypes.c_int64 * 5)()
    moc._check(lib().moc_linear_parts(PRODUCTS[product], rows, cin, cout, int(aligned), units, out), "moc_linear_parts")
    return Parts(out[0], bool(out[1]), *out[2:])
