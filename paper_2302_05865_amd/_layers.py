"""ctypes binding of the workers' backward pass (include/fa.h), same names as the C ABI.

The functions check tensor types and shapes, take torch's current stream of the tensors' device,
allocate outputs and workspace from torch's allocator (so a call is as safe on a side stream as
any torch operation) and forward to ``libfa.so``.  They are no autograd functions: what they
return has no graph, whether or not an input requires a gradient, and they put gradients where
they are told to.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from ._binding import _check, load_library
from ._ctypes_defs import FA_BF16, FA_CHECKPOINT_BLOCK, FA_ERR_ARG, FA_F32, FA_P_MAX


# What every call needs of torch and the library, looked up at the first one: small calls cost as much as their launches and
# what is done here.
torch = None
_CODES: dict = {}
_raw_stream = None
_lib = None


def _ready() -> None:
    global torch, _CODES, _raw_stream, _lib
    if _lib is not None:
        return
    import torch as _torch
    torch = _torch
    _CODES = {_torch.float32: FA_F32, _torch.bfloat16: FA_BF16}
    _raw_stream = getattr(_torch._C, "_cuda_getCurrentRawStream", None)
    if _raw_stream is None:
        def _raw_stream(index):
            return _torch.cuda.current_stream(index).cuda_stream
    _lib = load_library()


def _dtype(t, name: str) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16")
    return code


def _matrix(t, name: str, shape=None, like=None):
    """A [rows, width] device tensor with unit inner stride: (address, leading dimension)."""
    size, stride = t.shape, t.stride()
    if not t.is_cuda or len(size) != 2 or (stride[1] != 1 and size[1] > 1 and size[0] > 0):
        raise TypeError(f"{name} must be a two-dimensional device tensor with unit inner stride")
    if shape is not None and size != shape:
        raise TypeError(f"{name} must have shape {tuple(shape)}")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise TypeError(f"{name} must have the type and device of the other activations")
    if size[0] > 1 and stride[0] < size[1]:
        raise TypeError(f"{name}: rows must not overlap")
    return t.data_ptr(), stride[0]


def _vector(t, name: str, n: int, device, dtype=None):
    if t is None:
        return None
    if t.device != device or t.shape != (n,) or not t.is_contiguous() or (dtype is not None and t.dtype != dtype):
        raise TypeError(f"{name} must be a contiguous vector of {n} elements on {device}"
                        + (f" of {dtype}" if dtype is not None else ""))
    return t.data_ptr()


def _params(gamma, beta, n: int, device):
    """(gamma, beta, their type): both in one type."""
    if gamma is None:
        return None, _vector(beta, "beta", n, device), FA_F32 if beta is None else _dtype(beta, "gamma and beta")
    if beta is not None and gamma.dtype != beta.dtype:
        raise TypeError("gamma and beta must have the same type")
    return _vector(gamma, "gamma", n, device), _vector(beta, "beta", n, device), _dtype(gamma, "gamma and beta")


def _sizes(sizes: Sequence[int], rows: int):
    p = len(sizes)
    if not 1 <= p <= FA_P_MAX:
        raise TypeError(f"sizes must name 1 to {FA_P_MAX} workers")
    sizes = [int(k) for k in sizes]
    if min(sizes) < 0 or sum(sizes) != rows:
        raise TypeError(f"sizes must be the workers' numbers of rows, {rows} in all")
    return (ctypes.c_int64 * p)(*sizes), p


def _call(name: str, device, *args) -> None:
    """The library's function on torch's current stream of the device that the tensors are on."""
    index = device.index
    if index == torch.cuda.current_device():
        status = getattr(_lib, name)(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            status = getattr(_lib, name)(*args, _raw_stream(index))
    if status:
        _check(status, name)


class Checkpoint:
    """An activation [rows, features] in 8 bits: ``codes`` (int8, rows padded to whole blocks of
    32 features) and ``exponents`` (uint8, one for each block, rows padded to multiples of four).
    ``codes * 2**(exponents - 127)`` are its values, exponents 1 to 248, and NaN where the
    exponent is 255; the layout is that of include/fa.h."""

    __slots__ = ("codes", "exponents", "features")

    def __init__(self, codes, exponents, features: int):
        _ready()
        features = int(features)
        if features < 1:
            raise TypeError("features must be at least 1")
        pitch = -(-features // FA_CHECKPOINT_BLOCK) * FA_CHECKPOINT_BLOCK
        epitch = -(-features // (4 * FA_CHECKPOINT_BLOCK)) * 4
        if (codes.dim() != 2 or codes.dtype != torch.int8 or not codes.is_cuda or not codes.is_contiguous() or
                codes.shape[1] != pitch):
            raise TypeError(f"codes must be a contiguous [rows, {pitch}] int8 device tensor")
        if (exponents.dtype != torch.uint8 or exponents.device != codes.device or not exponents.is_contiguous() or
                tuple(exponents.shape) != (codes.shape[0], epitch)):
            raise TypeError(f"exponents must be a contiguous [{codes.shape[0]}, {epitch}] uint8 tensor beside codes")
        self.codes, self.exponents, self.features = codes, exponents, features

    @classmethod
    def empty(cls, rows: int, features: int, device="cuda") -> "Checkpoint":
        _ready()
        rows, features = int(rows), int(features)
        if rows < 0 or features < 1:
            raise TypeError("rows must be at least 0 and features at least 1")
        pitch = -(-features // FA_CHECKPOINT_BLOCK) * FA_CHECKPOINT_BLOCK
        epitch = -(-features // (4 * FA_CHECKPOINT_BLOCK)) * 4
        made = cls.__new__(cls)
        made.codes = torch.empty((rows, pitch), dtype=torch.int8, device=device)
        made.exponents = torch.empty((rows, epitch), dtype=torch.uint8, device=device)
        made.features = features
        return made

    @property
    def rows(self) -> int:
        return self.codes.shape[0]

    def _for(self, rows: int, features: Optional[int], device):
        if self.rows != rows or (features is not None and self.features != features) or self.codes.device != device:
            raise TypeError(f"the checkpoint is of [{self.rows}, {self.features}] on {self.codes.device}")
        return self.codes.data_ptr(), self.exponents.data_ptr()


def _apart(out, name: str, *others) -> None:
    for t in others:
        if t is not None and out.data_ptr() == t.data_ptr() and out.numel():
            raise TypeError(f"{name} must not overlap an input")


def fa_checkpoint_pack(x, out: Optional[Checkpoint] = None) -> Checkpoint:
    """``x`` [rows, features] in 8 bits."""
    _ready()
    ptr, ld = _matrix(x, "x")
    rows, features = x.shape
    dtype, device = _dtype(x, "x"), x.device
    if out is None:
        out = Checkpoint.empty(rows, features, device)
    codes, exponents = out._for(rows, features, device)
    _call("fa_checkpoint_pack", device, ptr, ld, rows, features, dtype, codes, exponents)
    return out


def fa_checkpoint_unpack(checkpoint: Checkpoint, dtype=None, out=None):
    """The values of a checkpoint as a [rows, features] tensor of ``dtype`` (default float32)."""
    _ready()
    rows, features = checkpoint.rows, checkpoint.features
    device = checkpoint.codes.device
    if out is None:
        out = torch.empty((rows, features), dtype=dtype or torch.float32, device=device)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError(f"out must be of {dtype}")
    ptr, ld = _matrix(out, "out", (rows, features))
    codes, exponents = checkpoint._for(rows, features, out.device)
    _call("fa_checkpoint_unpack", device, codes, exponents, rows, features, _dtype(out, "out"), ptr, ld)
    return out


def fa_layer_norm(x, gamma=None, beta=None, eps: float = 1e-5, checkpoint: Optional[Checkpoint] = None,
                  out=None, stats: bool = True):
    """``(y, mean, rstd)`` of the layer norm of every row of ``x`` [rows, features].  ``checkpoint``
    (``Checkpoint.empty(rows, features)``) receives the normalised rows, before gamma and beta, in
    8 bits.  ``stats=False``: mean and rstd are not wanted, and None."""
    _ready()
    ptr, ld = _matrix(x, "x")
    rows, features = x.shape
    dtype, device = _dtype(x, "x"), x.device
    g, b, param_dtype = _params(gamma, beta, features, device)
    if out is None:
        out = torch.empty((rows, features), dtype=x.dtype, device=device)
        yptr, ldy = out.data_ptr(), features
    else:
        yptr, ldy = _matrix(out, "out", (rows, features), x)
        _apart(out, "out", x)
    codes = exponents = mean = rstd = mptr = rptr = None
    if checkpoint is not None:
        codes, exponents = checkpoint._for(rows, features, device)
    if stats:
        mean = torch.empty(rows, dtype=torch.float32, device=device)
        rstd = torch.empty(rows, dtype=torch.float32, device=device)
        mptr, rptr = mean.data_ptr(), rstd.data_ptr()
    _call("fa_layer_norm", device, ptr, ld, rows, features, dtype, g, b, param_dtype, eps, yptr, ldy, mptr, rptr, codes,
          exponents)
    return out, mean, rstd


def fa_layer_norm_backward(dy, rstd, sizes: Sequence[int], dgamma=None, dbeta=None, *, gamma=None, x=None, mean=None,
                           checkpoint: Optional[Checkpoint] = None, residual=None, out=None):
    """dx of the layer norm, and in place every worker's ``dgamma[w]`` and ``dbeta[w]`` ([p, features],
    usually slices of G's rows).  ``sizes[w]``: rows of worker w.  The normalised rows come from the
    ``checkpoint`` or from ``x`` and ``mean``.  ``residual`` is added to dx."""
    _ready()
    ptr, ld = _matrix(dy, "dy")
    shape = dy.shape
    rows, features = shape
    dtype, device = _dtype(dy, "dy"), dy.device
    sz, p = _sizes(sizes, rows)
    if (x is None) == (checkpoint is None) or (x is not None and mean is None):
        raise TypeError("the normalised rows come from x and mean, or from checkpoint")
    if rstd is None:
        raise TypeError("rstd must be given")
    xptr, ldx = _matrix(x, "x", shape, dy) if x is not None else (None, 0)
    rptr, ldr = _matrix(residual, "residual", shape, dy) if residual is not None else (None, 0)
    codes, exponents = checkpoint._for(rows, features, device) if checkpoint is not None else (None, None)
    g, _, param_dtype = _params(gamma, None, features, device)
    mptr = _vector(mean, "mean", rows, device, torch.float32)
    sptr = _vector(rstd, "rstd", rows, device, torch.float32)
    if out is None:
        out = torch.empty(shape, dtype=dy.dtype, device=device)
        optr, ldo = out.data_ptr(), features
    else:
        optr, ldo = _matrix(out, "out", shape, dy)
        _apart(out, "out", dy, x, residual)
    grad, dgptr, lddg, dbptr, lddb = None, None, 0, None, 0
    if dgamma is not None:
        dgptr, lddg = _matrix(dgamma, "dgamma", (p, features))
        grad = dgamma
    if dbeta is not None:
        dbptr, lddb = _matrix(dbeta, "dbeta", (p, features), dgamma)
        grad = dbeta
    need, space, grad_dtype = 0, None, FA_F32
    if grad is not None:
        if grad.device != device:
            raise TypeError("dgamma and dbeta must be on the device of dy")
        grad_dtype = _dtype(grad, "dgamma and dbeta")
        need = _lib.fa_layer_norm_backward_workspace(sz, p, features)
        if need < 0:
            _check(FA_ERR_ARG, "fa_layer_norm_backward_workspace")
        if need:
            space = torch.empty(need, dtype=torch.uint8, device=device)
    _call("fa_layer_norm_backward", device, ptr, ld, sz, p, features, dtype, xptr, ldx, mptr, sptr, codes, exponents, g,
          param_dtype, rptr, ldr, optr, ldo, dgptr, lddg, dbptr, lddb, grad_dtype, space.data_ptr() if need else None, need)
    return out


def fa_linear_grad(dy, checkpoint: Checkpoint, sizes: Sequence[int], dweight, dbias=None, *, gamma=None, beta=None) -> None:
    """In place every worker's ``dweight[w]`` ([p, outputs, features], each [outputs, features]
    contiguous, usually slices of G's rows) and ``dbias[w]`` ([p, outputs]) of a linear layer from
    the gradient ``dy`` [rows, outputs] of its outputs and the checkpoint of its input.  With
    ``gamma`` and ``beta`` the layer's input was ``values * gamma + beta``."""
    _ready()
    ptr, ld = _matrix(dy, "dy")
    rows, outputs = dy.shape
    dtype, device, features = _dtype(dy, "dy"), dy.device, checkpoint.features
    sz, p = _sizes(sizes, rows)
    codes, exponents = checkpoint._for(rows, None, device)
    if (gamma is None) != (beta is None):
        raise TypeError("gamma and beta go together")
    g, b, param_dtype = _params(gamma, beta, features, device)
    stride = dweight.stride()
    if (dweight.device != device or dweight.shape != (p, outputs, features) or (features > 1 and stride[2] != 1) or
            (outputs > 1 and stride[1] != features) or (p > 1 and stride[0] < outputs * features)):
        raise TypeError(f"dweight must be [{p}, {outputs}, {features}] on {device}, every worker's part contiguous")
    bptr, ldb = None, 0
    if dbias is not None:
        bptr, ldb = _matrix(dbias, "dbias", (p, outputs), dweight)
    need, space = _lib.fa_linear_grad_workspace(sz, p, features, outputs, dtype), None
    if need < 0:
        _check(FA_ERR_ARG, "fa_linear_grad_workspace")
    if need:
        space = torch.empty(need, dtype=torch.uint8, device=device)
    _call("fa_linear_grad", device, ptr, ld, sz, p, features, outputs, dtype, codes, exponents, g, b, param_dtype,
          dweight.data_ptr(), stride[0], bptr, ldb, _dtype(dweight, "dweight"), space.data_ptr() if need else None, need)
