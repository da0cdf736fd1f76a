"""Python binding of the operators that a rematerialisation plan is run with (C ABI in
include/moccasin_training.h, in the same library as the evaluator).

Argument marshalling only, as in `moccasin`: tensors are checked and turned into descriptors (natively,
binding/training.cpp), results and workspaces are torch tensors, everything is asynchronous on `stream`
(default: torch's current stream) on the current device, where the tensors have to be.  Matrices are
two-dimensional CUDA tensors whose values of a row lie next to each other; rows may be any distance apart.  An `out` or `keep` that shares memory with an input is refused; it may be x of
moc_norm_forward, dy, x or residual of moc_norm_backward, residual of moc_linear_forward and pre of
moc_linear_backward_input themselves (same type and strides).  There is no CPU fallback: a missing library or GPU raises.

No call records a graph: results never require gradients, those of tensors that do included.  The gradients are calls of their
own (moc_*_backward*); inside torch's autograd they belong into the backward of a torch.autograd.Function.  What a call is given to
write to (parameters, moments, an `out`, a `keep`) counts as changed in place: autograd refuses a graph that has saved it before.  A captured
graph's replay changes memory that torch does not hear of.

A `Checkpoint` is an activation kept in 8 bits: a byte a value and a scale for 32 columns of a row.
"""
from __future__ import annotations

import collections
import ctypes
import typing

from . import moccasin as moc

MOC_TRAINING_VERSION = 3
MOC_F32, MOC_F16, MOC_BF16, MOC_E4M3, MOC_I8 = range(5)
FORMATS = {"e4m3": MOC_E4M3, "int8": MOC_I8}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
PRODUCTS = {"forward": 0, "backward_input": 1, "backward_weight": 2}
BLOCK = 32

EXPORTS = ("moc_checkpoint_write", "moc_checkpoint_read", "moc_norm_forward", "moc_norm_backward", "moc_norm_backward_work", "moc_linear_forward",
           "moc_linear_backward_input", "moc_linear_backward_weight", "moc_linear_work", "moc_linear_parts",
           "moc_residual_forward", "moc_residual_backward", "moc_residual_backward_work", "moc_logprob_forward_work", "moc_logprob_forward", "moc_logprob_backward", "moc_adamw_step", "moc_moments_read", "moc_training_version")


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


class Moments:
    """A tensor's two moments: float32 `m` and `v`, or in 8 bits uint8 `m` and `v` of as many values, and the scales of 32 of
    them each, uint8 `m_scales` and `v_scales`."""

    __slots__ = ("m", "v", "m_scales", "v_scales")

    def __init__(self, m, v, m_scales=None, v_scales=None):
        self.m, self.v, self.m_scales, self.v_scales = m, v, m_scales, v_scales

    @property
    def nbytes(self):
        return sum(x.numel() * x.element_size() for x in (self.m, self.v, self.m_scales, self.v_scales) if x is not None)


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
        for name, args in (("moc_norm_backward_work", [I64, I64]), ("moc_linear_work", [I64, I64, I64]), ("moc_residual_backward_work", [I64, I64, I64]),
                           ("moc_logprob_forward_work", [I64, I64, I32])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, I64
        for name, args in (("moc_residual_forward", [I64, I64, M, M, M, I64, F32, VP, VP, M, M, M, VP]),
                           ("moc_residual_backward", [I64, I64, M, M, M, M, M, I64, F32, VP, VP, M, M, VP, VP, I64, VP]), ("moc_logprob_forward", [I64, I64, M, VP, I32, F32, I32, VP, VP, VP, VP, VP, VP, I64, VP]),
                           ("moc_logprob_backward", [I64, I64, M, VP, VP, VP, I32, VP, VP, F32, M, VP]), ("moc_adamw_step", [I64, VP, VP, VP]), ("moc_moments_read", [I64, VP, VP])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, ctypes.c_int
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


class Norm(typing.NamedTuple):
    """A norm of rows: `kind` "layer" (mean and deviation, gamma and beta) or "rms" (the root of the mean square, gamma);
    None for gamma and beta stands for 1 and 0."""
    kind: str
    gamma: object = None
    beta: object = None
    eps: float = 1e-5


Residual = collections.namedtuple("Residual", "r n after before kept")
ResidualGrads = collections.namedtuple("ResidualGrads", "dx dblock gate after_gamma after_beta before_gamma before_beta")


def moc_residual_forward(x, block, gate=None, scale=1.0, after=None, before=None, keep=None, dtype=None, want_stream=True, out=None, out_norm=None, stream=None):
    """The stream between two blocks, r = scale * x + gate * after(block), and the norm before the next one, n = before(r): `after` and
    `before` are Norms or None, `gate` [cols] or [gates, cols] for rows / gates rows each, `block` a tensor or a Checkpoint, `x` may be
    None.  Returns (r, n, (mean, rstd) of each norm, n in 8 bits if `keep` names a format or is a Checkpoint to write to); None for
    what is not there.  `dtype`: n's, default the block's, or x's if that is a Checkpoint; r is of x's, or else the block's.  `out` may be x or block, and so may `out_norm`."""
    code, r, n, after, before, kept = _call("residual_forward", stream, x, block, gate, scale, after, before, keep, dtype, want_stream, out, out_norm)
    moc._check(code, "moc_residual_forward")
    return Residual(r, n, after, before, kept)


def moc_residual_backward(dr, dn, r=None, block=None, gate=None, scale=1.0, after=None, after_stats=None, before=None, before_stats=None, want_x=True, want_params=True, dtype=None,
                          out_x=None, out_block=None, work=None, stream=None):
    """The gradients of moc_residual_forward from those of the stream (or None) and of the norm (None without `before`), what the
    forward pass was given and what it has left; `r` and `block` are tensors or Checkpoints.  Returns (dx, dblock of `dtype`, default the
    block's, and float32 gradients of the gate, [gates, cols], and of the norms' parameters); None for what is not there.
    `out_x` may be dr or r, `out_block` dn or block."""
    code, *got = _call("residual_backward", stream, dr, dn, r, block, gate, scale, after, after_stats, before, before_stats, want_x, want_params, dtype, out_x, out_block, work)
    moc._check(code, "moc_residual_backward")
    return ResidualGrads(*got)


LogProbs = collections.namedtuple("LogProbs", "logp lse entropy top_logp top_tokens")


def moc_logprob_forward(logits, tokens=None, scale=1.0, top=0, work=None, stream=None):
    """Log probabilities of the rows of `logits` times `scale`: (logp of `tokens` (int32 or int64 [rows]; below 0: none), lse, entropy, float32
    [rows]; log probabilities and columns of the `top` most likely ones, float32 and int64 [rows, top]); None for what is not
    asked for."""
    code, *out = _call("logprob_forward", stream, logits, tokens, scale, top, work)
    moc._check(code, "moc_logprob_forward")
    return LogProbs(*out)


def moc_logprob_backward(logits, lse, tokens=None, dlogp=None, entropy=None, dentropy=None, scale=1.0, dtype=None, out=None, stream=None):
    """The gradient with regard to the logits from those of logp and of the entropy, float32 [rows], and what the forward pass has
    left.  `dtype`: the logits' (default) or float32; `out` may be the logits."""
    code, out = _call("logprob_backward", stream, logits, lse, tokens, dlogp, entropy, dentropy, scale, dtype, out)
    moc._check(code, "moc_logprob_backward")
    return out


def zero_moments(param, bits=8):
    """Moments of zeros for a parameter, in 32 or 8 bits a value."""
    torch = moc._tc()
    if bits not in (8, 32):
        raise ValueError(f"bits {bits!r}: expected 8 or 32")
    dtype = torch.float32 if bits == 32 else torch.uint8
    scales = lambda: torch.zeros(-(-param.numel() // BLOCK), dtype=torch.uint8, device=param.device) if bits == 8 else None   # noqa: E731
    return Moments(*(torch.zeros(param.shape, dtype=dtype, device=param.device) for _ in range(2)), scales(), scales())


def moc_adamw_step(params, grads, moments, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, copies=None, grad_scale=None, seed=0, stream=None):
    """A step of AdamW over many tensors, in place: `params`, `moments` (a Moments each) and `copies`, whose items are float16 or
    bfloat16 tensors for the parameters' new values, or None.  Tensors are contiguous.  `step` counts from 1; `weight_decay`
    is a number, or one for each tensor; gradients are taken times `grad_scale`.  `lr`, `step` and `grad_scale` may be CUDA tensors of one
    value (float32, int64, float32), which are read when the step runs: a captured call then finds each replay's own.
    `seed`: of the random bits that moments in 8 bits are rounded with (the step is mixed in, and each tensor's place in the call's list:
    calls for groups of parameters within a step need different seeds, or the groups' tensors are rounded by the same bits)."""
    code = _call("adamw_step", stream, params, grads, moments, copies, weight_decay, lr, step, *betas, eps, grad_scale, seed)
    moc._check(code, "moc_adamw_step")


def moc_moments_read(moments, dtype=None, out=None, stream=None):
    """[(m, v)..]: what the moments stand for, as tensors of `dtype` (default float32) or in those of `out`, pairs of tensors."""
    code, out = _call("moments_read", stream, moments, dtype, out)
    moc._check(code, "moc_moments_read")
    return out
