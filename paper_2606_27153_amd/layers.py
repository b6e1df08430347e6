"""Layer operators around the matrices the Muon step updates: a matrix product
with a fused epilogue (``linear``), the same grouped by expert
(``grouped_linear``) and ``layer_norm``, each with its backward pass; and those
at a model's ends and on the way to its experts: ``embedding``,
``linear_cross_entropy``, and ``sort_by_expert`` with ``dispatch`` and ``combine``.

Each operator comes as a function torch's autograd sees (``linear``,
``grouped_linear``, ``layer_norm``, ``embedding``, ``linear_cross_entropy``,
``dispatch``, ``combine``) and as its two passes (``*_forward``,
``*_backward``), which only enqueue HIP kernels on torch's current stream of the
tensors' device: no host synchronisation, no copies, nothing of the data kept
between calls.  Weights are [in, out] like the optimizer's workloads; the transposed
view of an [out, in] weight is taken as it lies.  Weight gradients come in the
weight's own memory layout, so that ``Muon`` steps them without a copy.

Tensors are fp32 or bf16 (one dtype per call; layer norm's weight and bias may be
fp32 next to bf16 activations), sums are fp32.  Rows may be strided (a slice of
wider rows), their elements may not.  Tokens, targets and experts come as int32 or
int64 numbers on the GPU, which the host never reads: one outside its range
stands for nobody (no table row, no target, no expert).  A bad argument raises ValueError or
TypeError before anything is launched; a number that the library refuses (eps, sizes
out of its range) MuonError.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional, Sequence, Union

import torch

from . import _layers_lib as LL
from ._lib import MUON_BF16, MUON_F32

_DTYPES = {torch.float32: MUON_F32, torch.bfloat16: MUON_BF16}
_lib = None


def _load():
    global _lib
    if _lib is None:
        _lib = LL.load()
    return _lib


def _compiled():
    """The operators of few bytes, called by compiled code; each returns None where an
    argument does not fit, and the function below of that name says which."""
    return LL._binding or LL.binding()


def _tensor(t, name: str) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor, not {type(t).__name__}")


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16")
    return code


def _rows(t: torch.Tensor, name: str, like: torch.Tensor, rows: Optional[int], cols: int):
    """(pointer, leading dimension) of a 2-D tensor whose rows are contiguous."""
    if t is not like:
        _tensor(t, name)
    if t.dim() != 2 or t.size(1) != cols or (rows is not None and t.size(0) != rows):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected ({'rows' if rows is None else rows}, {cols})")
    if t is not like:
        _same(t, name, like)
    ld, step = t.stride()
    if step != 1 and cols != 1:
        raise ValueError(f"{name}'s rows are not contiguous (stride {t.stride()})")
    if ld < cols:
        if t.size(0) > 1:
            raise ValueError(f"{name}'s rows overlap (stride {t.stride()})")
        ld = cols
    return t.data_ptr(), ld


def _same(t: torch.Tensor, name: str, like: torch.Tensor) -> None:
    if t.dtype != like.dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {like.dtype}")
    if t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, expected {like.device}")


def _vector(t: Optional[torch.Tensor], name: str, like: torch.Tensor, n: int):
    if t is None:
        return None
    _tensor(t, name)
    if t.dim() != 1 or t.size(0) != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous vector of {n} elements")
    _same(t, name, like)
    return t.data_ptr()


def _weight(w: torch.Tensor, like: torch.Tensor, inner: int):
    """(pointer, leading dimension, transposed, outer) of a weight [inner, outer]
    kept by rows, or by columns (the transposed view of an [outer, inner] one)."""
    _tensor(w, "weight")
    if w.dim() != 2 or w.size(0) != inner:
        raise ValueError(f"weight has shape {tuple(w.shape)}, expected ({inner}, out)")
    _same(w, "weight", like)
    outer = w.size(1)
    ld, step = w.stride()
    if (step == 1 or outer == 1) and (ld >= outer or inner == 1):
        return w.data_ptr(), max(ld, outer), 0, outer
    if (ld == 1 or inner == 1) and (step >= inner or outer == 1):
        return w.data_ptr(), max(step, inner), 1, outer
    raise ValueError(f"neither the rows nor the columns of the weight are contiguous (stride {w.stride()})")


def _input(x: torch.Tensor, name: str = "x") -> None:
    _tensor(x, name)
    if x.dim() != 2:
        raise ValueError(f"{name} must be 2-D [rows, features], got shape {tuple(x.shape)}")
    if not x.is_cuda:
        raise ValueError(f"{name} is not on a GPU")
    if x.size(1) == 0:
        raise ValueError(f"{name} has no features")


def _activation(name: str) -> int:
    code = LL.ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"unknown activation {name!r}; choose from {tuple(LL.ACTIVATIONS)}")
    return code


def _on_device(fn):
    """Runs fn with its first tensor's device current (which it nearly always is)."""
    @functools.wraps(fn)
    def run(*args, **kwargs):
        t = args[0] if args else next((v for v in kwargs.values() if isinstance(v, torch.Tensor)), None)
        index = t.device.index if isinstance(t, torch.Tensor) else None
        if index is None or index == torch._C._cuda_getDevice():
            return fn(*args, **kwargs)
        with torch.cuda.device(index):
            return fn(*args, **kwargs)
    return run


def _stream(t: torch.Tensor) -> int:
    """torch's current stream on the tensor's device."""
    return torch._C._cuda_getCurrentRawStream(t.device.index)


def _flags(backward: int, x: torch.Tensor, outer: int, *addresses: int) -> int:
    """Flags of the workspace functions: whether the pass is the backward one, and
    whether an operand's rows are off 16-byte chunks (addresses: pointers, and
    leading dimensions in bytes)."""
    size = x.element_size()
    bits = (x.size(1) * size) | (outer * size)
    for a in addresses:
        bits |= a
    return backward | (2 if bits & 15 else 0)


@functools.lru_cache(maxsize=4096)
def _bytes(name: str, *args) -> int:
    """What the library's workspace function says of these sizes."""
    n = ctypes.c_size_t()
    LL.check(getattr(_load(), name)(*args, ctypes.byref(n)))
    return n.value


def _workspace(n: int, like: torch.Tensor):
    """A workspace from torch's allocator: it belongs to the current stream, and
    goes back to it when the call that enqueued its use returns."""
    return like.new_empty((n,), dtype=torch.uint8) if n else None


# ------------------------------------------------------------------- linear

@_on_device
def linear_forward(x: torch.Tensor, weight: torch.Tensor, *, bias: Optional[torch.Tensor] = None,
                   residual: Optional[torch.Tensor] = None, activation: str = "none",
                   keep_preactivation: bool = False):
    """``act(x @ weight + bias) + residual`` for x [rows, in], weight [in, out].

    With ``keep_preactivation`` returns ``(y, z)``, z = x @ weight + bias being
    what ``linear_backward`` reads (None without an activation)."""
    lib = _load()
    _input(x)
    act = _activation(activation)
    code = _dtype_code(x)
    rows, inner = x.shape
    xp, ldx = _rows(x, "x", x, rows, inner)
    wp, ldw, wt, outer = _weight(weight, x, inner)
    if outer == 0:
        raise ValueError("weight has no output features")
    bp = _vector(bias, "bias", x, outer)
    rp, ldr = (None, 0) if residual is None else _rows(residual, "residual", x, rows, outer)
    stream = _stream(x)
    y = x.new_empty((rows, outer))
    z = x.new_empty((rows, outer)) if keep_preactivation and act else None
    size = x.element_size()
    need = _bytes("muon_linear_workspace_bytes", rows, inner, outer, code, act,
                  _flags(0, x, outer, xp, ldx * size, wp, ldw * size))
    ws = _workspace(need, x)
    LL.check(lib.muon_linear_forward(xp, ldx, wp, ldw, wt, bp, rp, ldr, y.data_ptr(), outer,
                                     None if z is None else z.data_ptr(), outer, rows, inner, outer, code, act,
                                     None if ws is None else ws.data_ptr(), need, stream))
    return (y, z) if keep_preactivation else y


def _like_weight(weight: torch.Tensor, transposed: int) -> torch.Tensor:
    """An uninitialised gradient in the weight's own layout, dense."""
    if transposed:
        return weight.new_empty((weight.size(1), weight.size(0))).t()
    return weight.new_empty(tuple(weight.shape))


@_on_device
def linear_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, *,
                    preactivation: Optional[torch.Tensor] = None, activation: str = "none", bias_grad: bool = False,
                    input_grad: bool = True, weight_grad: bool = True):
    """Gradients ``(dx, dweight, dbias)`` of ``linear_forward`` for the output
    gradient dy (the residual's gradient is dy); those not asked for are None.
    dweight is kept like the weight (by rows or by columns)."""
    lib = _load()
    _input(x)
    act = _activation(activation)
    code = _dtype_code(x)
    rows, inner = x.shape
    xp, ldx = _rows(x, "x", x, rows, inner)
    wp, ldw, wt, outer = _weight(weight, x, inner)
    if outer == 0:
        raise ValueError("weight has no output features")
    gp, ldg = _rows(dy, "dy", x, rows, outer)
    zp, ldz = None, 0
    if act:
        if preactivation is None:
            raise ValueError(f"the backward pass of {activation!r} needs the forward pass's preactivation")
        zp, ldz = _rows(preactivation, "preactivation", x, rows, outer)
    stream = _stream(x)
    dx = x.new_empty((rows, inner)) if input_grad else None
    dw = _like_weight(weight, wt) if weight_grad else None
    db = x.new_empty((outer,)) if bias_grad else None
    size = x.element_size()
    need = _bytes("muon_linear_workspace_bytes", rows, inner, outer, code, act,
                  _flags(1, x, outer, xp, ldx * size, wp, ldw * size, gp, ldg * size))
    ws = _workspace(need, x)
    LL.check(lib.muon_linear_backward(gp, ldg, xp, ldx, wp, ldw, wt, zp, ldz,
                                      None if dx is None else dx.data_ptr(), inner,
                                      None if dw is None else dw.data_ptr(), inner if wt else outer,
                                      None if db is None else db.data_ptr(), rows, inner, outer, code, act,
                                      None if ws is None else ws.data_ptr(), need, stream))
    return dx, dw, db


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, activation, grad_mode):
        # needs_input_grad says what requires a gradient, also where none is taken
        need = grad_mode and any(ctx.needs_input_grad[:3])
        y, z = linear_forward(x, weight, bias=bias, residual=residual, activation=activation,
                              keep_preactivation=True) if need else \
            (linear_forward(x, weight, bias=bias, residual=residual, activation=activation), None)
        ctx.activation = activation
        ctx.save_for_backward(x, weight, z)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, z = ctx.saved_tensors
        nx, nw, nb, nr = ctx.needs_input_grad[:4]
        dx = dw = db = None
        if nx or nw or nb:
            dx, dw, db = linear_backward(_once(dy), x, weight, preactivation=z, activation=ctx.activation,
                                         bias_grad=nb, input_grad=nx, weight_grad=nw)
        return dx, dw, db, dy if nr else None, None, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
           activation: str = "none", residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``act(x @ weight + bias) + residual`` over the last dimension of x,
    differentiable once.  weight is [in, out] (or the transposed view of an
    [out, in] one); activation is "none", "relu", "gelu", "gelu_tanh" or "silu"."""
    x2 = _flat(x, "x")
    lead = x.shape[:-1]
    r2 = None
    if residual is not None:
        r2 = _flat(residual, "residual")
        if residual.shape[:-1] != lead:   # (as many rows in another order are other rows)
            raise ValueError(f"residual has leading dimensions {tuple(residual.shape[:-1])}, x has {tuple(lead)}")
    y = _Linear.apply(x2, weight, bias, r2, activation, torch.is_grad_enabled())
    return y if x.dim() == 2 else y.view(*lead, y.shape[-1])


def _dense(t: torch.Tensor) -> torch.Tensor:
    """t, copied if its rows are not contiguous or overlap."""
    if t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= t.size(1):
        return t
    return t.contiguous()


def _flat(t: torch.Tensor, name: str) -> torch.Tensor:
    """t as dense rows of its last dimension."""
    if not isinstance(t, torch.Tensor):
        _tensor(t, name)
    if t.dim() != 2:
        if t.dim() == 0 or t.size(-1) == 0:
            raise ValueError(f"{name} has no features, its shape is {tuple(t.shape)}")
        t = t.reshape(-1, t.size(-1))
    return _dense(t)


def _once(dy: torch.Tensor) -> torch.Tensor:
    """A gradient for both products that read it: as it lies, or copied here where
    each of them would have to (rows off 16-byte chunks)."""
    dy = _dense(dy)
    if (dy.stride(0) * dy.element_size() | dy.data_ptr()) & 15:
        return dy.contiguous()
    return dy


# ----------------------------------------------------------- grouped linear

Weights = Union[torch.Tensor, Sequence[torch.Tensor]]


def _steps(t: torch.Tensor):
    """The strides that say where elements lie: those of more than one."""
    return [s for s, n in zip(t.stride(), t.shape) if n > 1]


def _experts(weights: Weights, like: torch.Tensor, inner: int):
    """(pointers, leading dimension, transposed, outer, count) of the experts'
    weights: one [experts, in, out] tensor or a sequence of [in, out] ones."""
    if isinstance(weights, torch.Tensor):
        if weights.dim() != 3:
            raise ValueError(f"weights must be [experts, in, out], got shape {tuple(weights.shape)}")
        n = weights.size(0)
        if n < 1 or n > LL.MUON_GROUPED_MAX_EXPERTS:
            raise ValueError(f"{n} experts; 1 to {LL.MUON_GROUPED_MAX_EXPERTS} are supported")
        p, ld, t, outer = _weight(weights[0], like, inner)
        step = weights.stride(0) * weights.element_size()
        return [p + i * step for i in range(n)], ld, t, outer, n
    n = len(weights)
    if n < 1 or n > LL.MUON_GROUPED_MAX_EXPERTS:
        raise ValueError(f"{n} experts; 1 to {LL.MUON_GROUPED_MAX_EXPERTS} are supported")
    p, ld, t, outer = _weight(weights[0], like, inner)
    first = weights[0]
    shape, stride, dtype, device = first.shape, first.stride(), like.dtype, like.device
    ptrs = [p]
    for i in range(1, n):   # (on every call: kept to what it takes)
        w = weights[i]
        if not isinstance(w, torch.Tensor):
            _tensor(w, f"weight {i}")
        if w.shape != shape or (w.stride() != stride and _steps(w) != _steps(first)):
            raise ValueError(f"weight {i} has shape {tuple(w.shape)} and stride {w.stride()}, the first one "
                             f"{tuple(shape)} and {stride}")
        if w.dtype != dtype or w.device != device:
            _same(w, f"weight {i}", like)
        ptrs.append(w.data_ptr())
    return ptrs, ld, t, outer, n


def _offsets(offsets: torch.Tensor, n: int, like: torch.Tensor) -> int:
    _tensor(offsets, "offsets")
    if offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.size(0) != n + 1 or offsets.stride(0) != 1:
        raise ValueError(f"offsets must be a contiguous int32 vector of {n + 1} elements")
    if offsets.device != like.device:
        raise ValueError(f"offsets is on {offsets.device}, expected {like.device}")
    return offsets.data_ptr()


@_on_device
def grouped_linear_forward(x: torch.Tensor, weights: Weights, offsets: torch.Tensor) -> torch.Tensor:
    """``y[t] = x[t] @ weights[e]`` for offsets[e] <= t < offsets[e + 1]: rows
    sorted by expert, int32 offsets on the GPU (the host never reads them).
    Rows outside every expert's range get 0."""
    lib = _load()
    _input(x)
    code = _dtype_code(x)
    rows, inner = x.shape
    xp, ldx = _rows(x, "x", x, rows, inner)
    ptrs, ldw, wt, outer, n = _experts(weights, x, inner)
    if outer == 0:
        raise ValueError("the weights have no output features")
    op = _offsets(offsets, n, x)
    stream = _stream(x)
    y = x.new_empty((rows, outer))
    size = x.element_size()
    need = _bytes("muon_grouped_linear_workspace_bytes", rows, inner, outer, n, code,
                  _flags(0, x, outer, xp, ldx * size, ldw * size, *ptrs))
    ws = _workspace(need, x)
    LL.check(lib.muon_grouped_linear_forward(xp, ldx, (ctypes.c_void_p * n)(*ptrs), ldw, wt, op, n, y.data_ptr(),
                                             outer, rows, inner, outer, code,
                                             None if ws is None else ws.data_ptr(), need, stream))
    return y


@_on_device
def grouped_linear_backward(dy: torch.Tensor, x: torch.Tensor, weights: Weights, offsets: torch.Tensor, *,
                            input_grad: bool = True, weight_grad: Union[bool, Sequence[bool]] = True):
    """Gradients ``(dx, dweights)`` of ``grouped_linear_forward``.  dweights is
    one [experts, in, out] tensor, or a list of its slices if the weights came
    as a sequence; an expert without rows gets zeros.  ``weight_grad`` may name
    per expert whether its gradient is wanted (None in the list if not)."""
    lib = _load()
    _input(x)
    code = _dtype_code(x)
    rows, inner = x.shape
    xp, ldx = _rows(x, "x", x, rows, inner)
    ptrs, ldw, wt, outer, n = _experts(weights, x, inner)
    if outer == 0:
        raise ValueError("the weights have no output features")
    gp, ldg = _rows(dy, "dy", x, rows, outer)
    op = _offsets(offsets, n, x)
    want = None
    if not isinstance(weight_grad, bool):
        want = [bool(v) for v in weight_grad]
        if len(want) != n:
            raise ValueError(f"weight_grad names {len(want)} experts, there are {n}")
        weight_grad = any(want)
    stream = _stream(x)
    dx = x.new_empty((rows, inner)) if input_grad else None
    dw = dptrs = None
    if weight_grad:
        a, b = (outer, inner) if wt else (inner, outer)
        dw = x.new_empty((n, a, b))
        step = a * b * dw.element_size()
        base = dw.data_ptr()
        dptrs = (ctypes.c_void_p * n)(*[base + i * step if want is None or want[i] else None for i in range(n)])
        if wt:
            dw = dw.transpose(1, 2)
    size = x.element_size()
    need = _bytes("muon_grouped_linear_workspace_bytes", rows, inner, outer, n, code,
                  _flags(1, x, outer, xp, ldx * size, ldw * size, gp, ldg * size, *ptrs))
    ws = _workspace(need, x)
    LL.check(lib.muon_grouped_linear_backward(gp, ldg, xp, ldx, (ctypes.c_void_p * n)(*ptrs), ldw, wt, op, n,
                                              None if dx is None else dx.data_ptr(), inner, dptrs,
                                              inner if wt else outer, rows, inner, outer, code,
                                              None if ws is None else ws.data_ptr(), need, stream))
    if dw is not None and (want is not None or not isinstance(weights, torch.Tensor)):
        dw = [dw[i] if want is None or want[i] else None for i in range(n)]
    return dx, dw


class _GroupedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, offsets, *weights):
        ctx.stacked = len(weights) == 1 and isinstance(weights[0], torch.Tensor) and weights[0].dim() == 3
        ctx.save_for_backward(x, offsets, *weights)
        return grouped_linear_forward(x, weights[0] if ctx.stacked else weights, offsets)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, offsets, *weights = ctx.saved_tensors
        nx, _, *nw = ctx.needs_input_grad
        if not (nx or any(nw)):
            return (None, None) + (None,) * len(weights)
        dx, dw = grouped_linear_backward(_dense(dy), x, weights[0] if ctx.stacked else weights, offsets,
                                         input_grad=nx, weight_grad=nw[0] if ctx.stacked else nw)
        if ctx.stacked:
            return dx, None, dw
        return (dx, None, *(dw if dw is not None else (None,) * len(weights)))


def grouped_linear(x: torch.Tensor, weights: Weights, offsets: torch.Tensor) -> torch.Tensor:
    """``y[t] = x[t] @ weights[e]`` for the rows offsets[e] <= t < offsets[e + 1]
    of x [rows, in], differentiable once.  weights: one [experts, in, out]
    tensor, or the experts' own [in, out] parameters (which ``Muon`` steps)."""
    _tensor(x, "x")
    ws = (weights,) if isinstance(weights, torch.Tensor) else tuple(weights)
    return _GroupedLinear.apply(_dense(x), offsets, *ws)


# --------------------------------------------------------------- layer norm

def _norm_vectors(x: torch.Tensor, vectors, cols: int):
    """Pointers of the weight and bias, and the dtype code they share."""
    code, ptrs = None, []
    for name, t in vectors:
        if t is None:
            ptrs.append(None)
            continue
        _tensor(t, name)
        if t.dim() != 1 or t.size(0) != cols or (cols > 1 and t.stride(0) != 1):
            raise ValueError(f"{name} must be a contiguous vector of {cols} elements")
        if t.device != x.device:
            raise ValueError(f"{name} is on {t.device}, expected {x.device}")
        if t.dtype not in (torch.float32, x.dtype):
            raise ValueError(f"{name} has dtype {t.dtype}, expected float32 or {x.dtype}")
        c = _DTYPES[t.dtype]
        if code is not None and c != code:
            raise ValueError("weight and bias have different dtypes")
        code = c
        ptrs.append(t.data_ptr())
    return (*ptrs, _DTYPES[x.dtype] if code is None else code)


@_on_device
def layer_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
                       eps: float = 1e-5, keep_stats: bool = False):
    """Layer norm over the columns of x [rows, cols].  With ``keep_stats``
    returns ``(y, mean, rstd)``, the fp32 statistics its backward pass reads."""
    lib = _load()
    _input(x)
    code = _dtype_code(x)
    rows, cols = x.shape
    xp, ldx = _rows(x, "x", x, rows, cols)
    wp, bp, wcode = _norm_vectors(x, (("weight", weight), ("bias", bias)), cols)
    eps = float(eps)
    stream = _stream(x)
    y = x.new_empty((rows, cols))
    mean = rstd = None
    if keep_stats:
        mean, rstd = x.new_empty((rows,), dtype=torch.float32), x.new_empty((rows,), dtype=torch.float32)
    LL.check(lib.muon_layer_norm_forward(xp, ldx, wp, bp, y.data_ptr(), cols,
                                         None if mean is None else mean.data_ptr(),
                                         None if rstd is None else rstd.data_ptr(), rows, cols, eps, code, wcode,
                                         stream))
    return (y, mean, rstd) if keep_stats else y


@_on_device
def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor,
                        rstd: torch.Tensor, *, input_grad: bool = True, weight_grad: bool = True,
                        bias_grad: bool = True, bias_dtype: Optional[torch.dtype] = None):
    """Gradients ``(dx, dweight, dbias)`` of ``layer_norm_forward``; those not
    asked for are None.  dweight and dbias have the weight's dtype; without a
    weight, ``bias_dtype`` (float32 or x's, which is the default)."""
    lib = _load()
    _input(x)
    code = _dtype_code(x)
    rows, cols = x.shape
    xp, ldx = _rows(x, "x", x, rows, cols)
    gp, ldg = _rows(dy, "dy", x, rows, cols)
    wp, _, wcode = _norm_vectors(x, (("weight", weight), ("bias", None)), cols)
    if weight is None and bias_dtype is not None:
        if bias_dtype not in (torch.float32, x.dtype):
            raise ValueError(f"bias_dtype {bias_dtype}, expected float32 or {x.dtype}")
        wcode = _DTYPES[bias_dtype]
    for name, t in (("mean", mean), ("rstd", rstd)):
        _tensor(t, name)
        if t.dtype != torch.float32 or t.dim() != 1 or t.size(0) != rows or (rows > 1 and t.stride(0) != 1):
            raise ValueError(f"{name} must be a contiguous float32 vector of {rows} elements")
        if t.device != x.device:
            raise ValueError(f"{name} is on {t.device}, expected {x.device}")
    stream = _stream(x)
    dx = x.new_empty((rows, cols)) if input_grad else None
    wdt = torch.float32 if wcode == MUON_F32 else x.dtype
    dw = x.new_empty((cols,), dtype=wdt) if weight_grad else None
    db = x.new_empty((cols,), dtype=wdt) if bias_grad else None
    need = _bytes("muon_layer_norm_workspace_bytes", rows, cols) if weight_grad or bias_grad else 0
    ws = _workspace(need, x)
    LL.check(lib.muon_layer_norm_backward(gp, ldg, xp, ldx, wp, mean.data_ptr(), rstd.data_ptr(),
                                          None if dx is None else dx.data_ptr(), cols,
                                          None if dw is None else dw.data_ptr(),
                                          None if db is None else db.data_ptr(), rows, cols, code, wcode,
                                          None if ws is None else ws.data_ptr(), need, stream))
    return dx, dw, db


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, grad_mode):
        if not (grad_mode and any(ctx.needs_input_grad[:3])):
            return layer_norm_forward(x, weight, bias, eps=eps)
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps=eps, keep_stats=True)
        ctx.bias_dtype = None if bias is None else bias.dtype
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        nx, nw, nb = ctx.needs_input_grad[:3]
        dx, dw, db = layer_norm_backward(_dense(dy), x, weight, mean, rstd, input_grad=nx, weight_grad=nw,
                                         bias_grad=nb, bias_dtype=ctx.bias_dtype)
        return dx, dw, db, None, None


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
               eps: float = 1e-5) -> torch.Tensor:
    """Layer norm over the last dimension of x, differentiable once."""
    y = _LayerNorm.apply(_flat(x, "x"), weight, bias, float(eps), torch.is_grad_enabled())
    return y if x.dim() == 2 else y.view(x.shape)


# ------------------------------------------------- tokens, targets, experts

_NUMBERS = {torch.int32: 4, torch.int64: 8}


def _numbers(t: torch.Tensor, name: str, shape=None, like: Optional[torch.Tensor] = None):
    """(pointer, bytes of an element) of a contiguous tensor of numbers."""
    _tensor(t, name)
    size = _NUMBERS.get(t.dtype)
    if size is None:
        raise TypeError(f"{name} has dtype {t.dtype}, expected int32 or int64")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} is not contiguous (stride {t.stride()})")
    if not t.is_cuda:
        raise ValueError(f"{name} is not on a GPU")
    if like is not None and t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, expected {like.device}")
    return t.data_ptr(), size


# ---------------------------------------------------------------- embedding

def embedding_forward(ids: torch.Tensor, weight: torch.Tensor, *, scale: float = 1.0) -> torch.Tensor:
    """``scale * weight[ids]`` for ids of any shape and a table [vocab, cols]; a
    number outside [0, vocab) gets a row of 0."""
    scale = float(scale)
    y = _compiled().embedding_forward(ids, weight, scale)
    return _embedding_forward(ids, weight, scale) if y is None else y


@_on_device
def _embedding_forward(ids: torch.Tensor, weight: torch.Tensor, scale: float) -> torch.Tensor:
    lib = _load()
    ip, size = _numbers(ids, "ids")
    _input(weight, "weight")
    code = _dtype_code(weight)
    vocab, cols = weight.shape
    if vocab == 0:
        raise ValueError("weight has no rows")
    _numbers(ids, "ids", None, weight)
    wp, ldw = _rows(weight, "weight", weight, vocab, cols)
    stream = _stream(weight)
    y = weight.new_empty((*ids.shape, cols))
    LL.check(lib.muon_embedding_forward(ip, size, wp, ldw, y.data_ptr(), cols, ids.numel(), vocab, cols, scale, code,
                                        stream))
    return y


def embedding_backward(dy: torch.Tensor, ids: torch.Tensor, vocab: int, *, scale: float = 1.0) -> torch.Tensor:
    """The table's gradient [vocab, cols] for the output gradient dy [*ids.shape,
    cols]: ``scale`` times the sum of each token's rows, taken in their order."""
    scale = float(scale)
    dw = _compiled().embedding_backward(dy, ids, vocab, scale)
    return _embedding_backward(dy, ids, vocab, scale) if dw is None else dw


@_on_device
def _embedding_backward(dy: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float) -> torch.Tensor:
    lib = _load()
    _tensor(dy, "dy")
    ip, size = _numbers(ids, "ids")
    if dy.dim() != ids.dim() + 1 or dy.shape[:-1] != ids.shape:
        raise ValueError(f"dy has shape {tuple(dy.shape)}, expected {(*ids.shape, 'cols')}")
    dy = _flat(dy, "dy")
    _input(dy, "dy")
    code = _dtype_code(dy)
    rows, cols = dy.shape
    _numbers(ids, "ids", None, dy)
    gp, ldg = _rows(dy, "dy", dy, rows, cols)
    vocab = int(vocab)
    if vocab < 1:
        raise ValueError(f"vocab {vocab}: a table has at least one row")
    stream = _stream(dy)
    dw = dy.new_empty((vocab, cols))
    need = _bytes("muon_embedding_workspace_bytes", rows, vocab, cols)
    ws = _workspace(need, dy)
    LL.check(lib.muon_embedding_backward(gp, ldg, ip, size, dw.data_ptr(), cols, rows, vocab, cols, scale, code,
                                         None if ws is None else ws.data_ptr(), need, stream))
    return dw


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, weight, scale):
        ctx.vocab, ctx.scale = weight.size(0), scale
        ctx.save_for_backward(ids)
        return embedding_forward(ids, weight, scale=scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        if not ctx.needs_input_grad[1]:
            return None, None, None
        return None, embedding_backward(dy, ctx.saved_tensors[0], ctx.vocab, scale=ctx.scale), None


def embedding(ids: torch.Tensor, weight: torch.Tensor, *, scale: float = 1.0) -> torch.Tensor:
    """``scale * weight[ids]``, differentiable once in the table [vocab, cols].  The
    table can be the transposed weight of ``linear_cross_entropy`` too."""
    _tensor(ids, "ids")
    _tensor(weight, "weight")
    return _Embedding.apply(ids.contiguous(), _dense(weight), float(scale))


# ----------------------------------------- tokens to their experts and back

class Routing(NamedTuple):
    """A router's choices sorted by expert (``sort_by_expert``)."""
    offsets: torch.Tensor    # int32 [experts + 1]: each expert's rows, as grouped_linear takes them
    position: torch.Tensor   # int32 [tokens, top]: each choice's row, -1 for one of no expert
    source: torch.Tensor     # int32 [tokens * top]: each row's choice t * top + j; behind the last, ~ those of no expert


def sort_by_expert(experts: torch.Tensor, count: int) -> Routing:
    """The choices experts [tokens, top] of ``count`` experts sorted by expert, in
    their own order within each.  One outside [0, count) goes to no expert."""
    found = _compiled().sort_by_expert(experts, count)
    return _sort_by_expert(experts, count) if found is None else Routing(*found)


@_on_device
def _sort_by_expert(experts: torch.Tensor, count: int) -> Routing:
    lib = _load()
    ip, size = _numbers(experts, "experts")
    if experts.dim() != 2:
        raise ValueError(f"experts must be [tokens, top], got shape {tuple(experts.shape)}")
    tokens, top = experts.shape
    count = int(count)
    for name, n in (("top", top), ("count", count)):
        if n < 1 or n > LL.MUON_GROUPED_MAX_EXPERTS:
            raise ValueError(f"{name} {n}; 1 to {LL.MUON_GROUPED_MAX_EXPERTS} are supported")
    stream = _stream(experts)
    i32 = torch.int32
    routing = Routing(experts.new_empty((count + 1,), dtype=i32), experts.new_empty((tokens, top), dtype=i32),
                      experts.new_empty((tokens * top,), dtype=i32))
    need = _bytes("muon_sort_by_expert_workspace_bytes", tokens, top)
    ws = _workspace(need, experts)
    LL.check(lib.muon_sort_by_expert(ip, size, tokens, top, count, routing.offsets.data_ptr(),
                                     routing.position.data_ptr(), routing.source.data_ptr(),
                                     None if ws is None else ws.data_ptr(), need, stream))
    return routing


def _routing(routing, like: torch.Tensor):
    """(pointer of position, of source, tokens, top)."""
    if not isinstance(routing, tuple) or len(routing) != 3:
        raise TypeError(f"routing must come from sort_by_expert, got {type(routing).__name__}")
    _, position, source = routing
    for t, name, dim in ((position, "position", 2), (source, "source", 1)):
        if not isinstance(t, torch.Tensor):
            _tensor(t, name)
        if t.dtype != torch.int32 or t.dim() != dim or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 tensor of {dim} dimensions")
        if t.device != like.device:
            raise ValueError(f"{name} is on {t.device}, expected {like.device}")
    tokens, top = position.shape
    if source.size(0) != tokens * top:
        raise ValueError(f"source has {source.size(0)} rows, position {tokens} x {top} choices")
    return position.data_ptr(), source.data_ptr(), tokens, top


def _router_weights(weights: torch.Tensor, x: torch.Tensor, tokens: int, top: int):
    _tensor(weights, "weights")
    if weights.shape != (tokens, top) or not weights.is_contiguous():
        raise ValueError(f"weights must be contiguous and [{tokens}, {top}], got shape {tuple(weights.shape)} and "
                         f"stride {weights.stride()}")
    if weights.device != x.device:
        raise ValueError(f"weights is on {weights.device}, expected {x.device}")
    if weights.dtype not in (torch.float32, x.dtype):
        raise ValueError(f"weights has dtype {weights.dtype}, expected float32 or {x.dtype}")
    return weights.data_ptr(), _DTYPES[weights.dtype]


def dispatch_forward(x: torch.Tensor, routing: Routing) -> torch.Tensor:
    """Every token's row x[t] at its choices' rows [tokens * top, cols], sorted by
    expert; rows behind the last expert's get 0."""
    rows = _compiled().dispatch_forward(x, routing)
    return _dispatch_forward(x, routing) if rows is None else rows


@_on_device
def _dispatch_forward(x: torch.Tensor, routing: Routing) -> torch.Tensor:
    lib = _load()
    _input(x)
    code = _dtype_code(x)
    pp, sp, tokens, top = _routing(routing, x)
    cols = x.size(1)
    xp, ldx = _rows(x, "x", x, tokens, cols)
    stream = _stream(x)
    rows = x.new_empty((tokens * top, cols))
    LL.check(lib.muon_dispatch_forward(xp, ldx, pp, sp, rows.data_ptr(), cols, tokens, top, cols, code, stream))
    return rows


def dispatch_backward(drows: torch.Tensor, routing: Routing) -> torch.Tensor:
    """dx [tokens, cols]: the sum of each token's choices' rows."""
    dx = _compiled().dispatch_backward(drows, routing)
    return _dispatch_backward(drows, routing) if dx is None else dx


@_on_device
def _dispatch_backward(drows: torch.Tensor, routing: Routing) -> torch.Tensor:
    lib = _load()
    _input(drows, "drows")
    code = _dtype_code(drows)
    pp, _, tokens, top = _routing(routing, drows)
    cols = drows.size(1)
    rp, ldr = _rows(drows, "drows", drows, tokens * top, cols)
    stream = _stream(drows)
    dx = drows.new_empty((tokens, cols))
    LL.check(lib.muon_dispatch_backward(rp, ldr, pp, dx.data_ptr(), cols, tokens, top, cols, code, stream))
    return dx


def combine_forward(rows: torch.Tensor, weights: torch.Tensor, routing: Routing, *,
                    residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``y[t] = residual[t] + sum of weights[t, j] * rows[position[t, j]]`` over the
    token's choices; weights [tokens, top] are fp32 or of the rows' dtype."""
    y = _compiled().combine_forward(rows, weights, routing, residual)
    return _combine_forward(rows, weights, routing, residual) if y is None else y


@_on_device
def _combine_forward(rows: torch.Tensor, weights: torch.Tensor, routing: Routing,
                     residual: Optional[torch.Tensor]) -> torch.Tensor:
    lib = _load()
    _input(rows, "rows")
    code = _dtype_code(rows)
    pp, _, tokens, top = _routing(routing, rows)
    cols = rows.size(1)
    rp, ldr = _rows(rows, "rows", rows, tokens * top, cols)
    wp, wcode = _router_weights(weights, rows, tokens, top)
    sp, lds = (None, 0) if residual is None else _rows(residual, "residual", rows, tokens, cols)
    stream = _stream(rows)
    y = rows.new_empty((tokens, cols))
    LL.check(lib.muon_combine_forward(rp, ldr, wp, wcode, pp, sp, lds, y.data_ptr(), cols, tokens, top, cols, code,
                                      stream))
    return y


def combine_backward(dy: torch.Tensor, rows: torch.Tensor, weights: torch.Tensor, routing: Routing, *,
                     rows_grad: bool = True, weights_grad: bool = True):
    """Gradients ``(drows, dweights)`` of ``combine_forward`` (the residual's is dy);
    those not asked for are None.  Rows behind the last expert's get 0."""
    found = _compiled().combine_backward(dy, rows, weights, routing, rows_grad, weights_grad)
    return _combine_backward(dy, rows, weights, routing, rows_grad, weights_grad) if found is None else found


@_on_device
def _combine_backward(dy: torch.Tensor, rows: torch.Tensor, weights: torch.Tensor, routing: Routing, rows_grad: bool,
                      weights_grad: bool):
    lib = _load()
    _input(dy, "dy")
    code = _dtype_code(dy)
    _, sp, tokens, top = _routing(routing, dy)
    cols = dy.size(1)
    gp, ldg = _rows(dy, "dy", dy, tokens, cols)
    rp, ldr = _rows(rows, "rows", dy, tokens * top, cols)
    wp, wcode = _router_weights(weights, dy, tokens, top)
    stream = _stream(dy)
    drows = dy.new_empty((tokens * top, cols)) if rows_grad else None
    dweights = torch.empty_like(weights) if weights_grad else None
    LL.check(lib.muon_combine_backward(gp, ldg, rp, ldr, wp, wcode, sp, None if drows is None else drows.data_ptr(),
                                       cols, None if dweights is None else dweights.data_ptr(), tokens, top, cols,
                                       code, stream))
    return drows, dweights


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, *routing):
        ctx.save_for_backward(*routing)
        return dispatch_forward(x, Routing(*routing))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, drows):
        dx = dispatch_backward(_dense(drows), Routing(*ctx.saved_tensors)) if ctx.needs_input_grad[0] else None
        return dx, None, None, None


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rows, weights, residual, *routing):
        ctx.save_for_backward(rows, weights, *routing)
        return combine_forward(rows, weights, Routing(*routing), residual=residual)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        rows, weights, *routing = ctx.saved_tensors
        nr, nw, ns = ctx.needs_input_grad[:3]
        drows = dweights = None
        if nr or nw:
            drows, dweights = combine_backward(_dense(dy), rows, weights, Routing(*routing), rows_grad=nr,
                                               weights_grad=nw)
        return drows, dweights, dy if ns else None, None, None, None


def dispatch(x: torch.Tensor, routing: Routing) -> torch.Tensor:
    """The rows [tokens * top, cols] that ``grouped_linear`` takes with
    ``routing.offsets``, differentiable once in x [tokens, cols]."""
    _tensor(x, "x")
    return _Dispatch.apply(_dense(x), *routing)


def combine(rows: torch.Tensor, weights: torch.Tensor, routing: Routing, *,
            residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The experts' outputs back at their tokens, weighted and added up (to the
    residual), differentiable once in rows, weights and residual."""
    _tensor(rows, "rows")
    _tensor(weights, "weights")
    if residual is not None:
        _tensor(residual, "residual")
        residual = _dense(residual)
    return _Combine.apply(_dense(rows), weights.contiguous(), residual, *routing)


# ------------------------------------------------------ linear cross entropy

def _reduction(name: str) -> int:
    code = LL.REDUCTIONS.get(name)
    if code is None:
        raise ValueError(f"unknown reduction {name!r}; choose from {tuple(LL.REDUCTIONS)}")
    return code


def _ignore(index) -> int:
    index = int(index)
    if not -1 << 63 <= index < 1 << 63:
        raise ValueError(f"ignore_index {index} does not fit in 64 bits")
    return index


def _loss_flags(backward: int, x: torch.Tensor, outer: int, xp: int, ldx: int, wp: int, ldw: int) -> int:
    """_flags, and room for the copies that rows far apart need too."""
    size = x.element_size()
    far = 2 if max(ldx, ldw) * size >= 1 << 23 else 0
    return _flags(backward, x, outer, xp, ldx * size, wp, ldw * size) | far


@_on_device
def linear_cross_entropy_forward(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, *,
                                 reduction: str = "mean", ignore_index: int = -100):
    """``(loss, lse)``: softmax cross entropy of the logits x @ weight for x [rows,
    in], weight [in, vocab], targets [rows], and the rows' log of the sum of
    exponentials, which the backward pass reads.  The logits are never kept: the
    vocabulary is gone through in pieces.  A row whose target is ignore_index or
    outside [0, vocab) has loss 0 and no gradients, whatever it holds, and does not
    count in the mean.  Both are fp32; loss is one number unless the reduction is "none"."""
    lib = _load()
    _input(x)
    red = _reduction(reduction)
    code = _dtype_code(x)
    rows, inner = x.shape
    xp, ldx = _rows(x, "x", x, rows, inner)
    wp, ldw, wt, outer = _weight(weight, x, inner)
    if outer == 0:
        raise ValueError("weight has no output features")
    tp, tsize = _numbers(targets, "targets", (rows,), x)
    ignore = _ignore(ignore_index)
    stream = _stream(x)
    lse = x.new_empty((rows,), dtype=torch.float32)
    loss = x.new_empty((rows,) if red == 0 else (), dtype=torch.float32)
    need = _bytes("muon_linear_cross_entropy_workspace_bytes", rows, inner, outer, code,
                  _loss_flags(0, x, outer, xp, ldx, wp, ldw))
    ws = _workspace(need, x)
    LL.check(lib.muon_linear_cross_entropy_forward(xp, ldx, wp, ldw, wt, tp, tsize, ignore, red, loss.data_ptr(),
                                                   lse.data_ptr(), rows, inner, outer, code,
                                                   None if ws is None else ws.data_ptr(), need, stream))
    return loss, lse


@_on_device
def linear_cross_entropy_backward(dloss: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                                  lse: torch.Tensor, *, reduction: str = "mean", ignore_index: int = -100,
                                  input_grad: bool = True, weight_grad: bool = True):
    """Gradients ``(dx, dweight)`` of ``linear_cross_entropy_forward`` for the
    loss's fp32 gradient (of its shape); those not asked for are None.  The logits
    are computed again, piece by piece.  dweight is kept like the weight."""
    lib = _load()
    _input(x)
    red = _reduction(reduction)
    code = _dtype_code(x)
    rows, inner = x.shape
    xp, ldx = _rows(x, "x", x, rows, inner)
    wp, ldw, wt, outer = _weight(weight, x, inner)
    if outer == 0:
        raise ValueError("weight has no output features")
    tp, tsize = _numbers(targets, "targets", (rows,), x)
    for name, t, shape in (("dloss", dloss, (rows,) if red == 0 else ()), ("lse", lse, (rows,))):
        _tensor(t, name)
        if t.dtype != torch.float32 or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 tensor of shape {shape}")
        if t.device != x.device:
            raise ValueError(f"{name} is on {t.device}, expected {x.device}")
    ignore = _ignore(ignore_index)
    stream = _stream(x)
    dx = x.new_empty((rows, inner)) if input_grad else None
    dw = _like_weight(weight, wt) if weight_grad else None
    need = _bytes("muon_linear_cross_entropy_workspace_bytes", rows, inner, outer, code,
                  _loss_flags(1, x, outer, xp, ldx, wp, ldw))
    ws = _workspace(need, x)
    LL.check(lib.muon_linear_cross_entropy_backward(dloss.data_ptr(), xp, ldx, wp, ldw, wt, tp, tsize, ignore, red,
                                                    lse.data_ptr(), None if dx is None else dx.data_ptr(), inner,
                                                    None if dw is None else dw.data_ptr(), inner if wt else outer,
                                                    rows, inner, outer, code,
                                                    None if ws is None else ws.data_ptr(), need, stream))
    return dx, dw


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, targets, reduction, ignore_index, grad_mode):
        loss, lse = linear_cross_entropy_forward(x, weight, targets, reduction=reduction, ignore_index=ignore_index)
        if grad_mode and any(ctx.needs_input_grad[:2]):
            ctx.how = dict(reduction=reduction, ignore_index=ignore_index)
            ctx.save_for_backward(x, weight, targets, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        x, weight, targets, lse = ctx.saved_tensors
        nx, nw = ctx.needs_input_grad[:2]
        dx, dw = linear_cross_entropy_backward(dloss.contiguous(), x, weight, targets, lse, input_grad=nx,
                                               weight_grad=nw, **ctx.how)
        return dx, dw, None, None, None, None


def linear_cross_entropy(x: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, *, reduction: str = "mean",
                         ignore_index: int = -100) -> torch.Tensor:
    """Softmax cross entropy of the logits x @ weight over the last dimension of x,
    without the logits, differentiable once in x and weight.  targets has x's
    leading dimensions; weight is [in, vocab], or the transposed view of an embedding
    table [vocab, in].  reduction is "mean" (over the rows with a target; 0 if there are
    none), "sum" or "none"."""
    x2 = _flat(x, "x")
    _tensor(targets, "targets")
    if targets.shape != x.shape[:-1]:
        raise ValueError(f"targets has shape {tuple(targets.shape)}, x has leading dimensions {tuple(x.shape[:-1])}")
    loss = _LinearCrossEntropy.apply(x2, weight, targets.reshape(-1).contiguous(), reduction, int(ignore_index),
                                     torch.is_grad_enabled())
    return loss.view(targets.shape) if reduction == "none" else loss
