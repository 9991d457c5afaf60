"""The dense operators beside the store: what a training step runs between a Get
and the apply of its gradients (MLKV, Section 2.1: N(w_nn; E(w_emb; x)); Figure 2).

    rows = store.get(keys)                                              # fp32 [n, d]
    h, stats = layer_norm(rows, g, b, out_dtype=torch.bfloat16, save_stats=True)
    y, pre = linear(h, w, bias, activation="silu", residual=h, save_pre=True)
    r = token_logprobs(linear(y, classes), targets, top=5)              # logprob, entropy, alternatives
    dz = token_logprobs_backward(logits, targets, r, dlogprob)
    dx, dw, db = linear_backward(dy, h, w, pre, activation="silu", bias=True)
    dx, dg, db = layer_norm_backward(dy, rows, g, stats)
    store.apply_grad(keys, dx)

Matrices are 2-d CUDA tensors of torch.float32, torch.bfloat16 or torch.float16
(the products: the last two) with any row stride; one whose rows are not
contiguous, or overlap, is copied first.  Every call is enqueued on the current
torch stream of its first tensor's device and runs in the CUDA library; working
memory comes from torch's allocator for the length of the call.  This module
only checks arguments (TypeError, ValueError) and passes pointers.  Formulas and
the treatment of masked and invalid values: include/mlkv_dense.h.
"""
import contextlib
import typing

import torch

from . import _lib as L
from .store import MLKVError, _stream

_TYPES = {torch.float32: L.TYPE_FLOAT, torch.bfloat16: L.TYPE_BFLOAT, torch.float16: L.TYPE_HALF}
_ACTIVATIONS = {None: L.ACT_NONE, "none": L.ACT_NONE, "relu": L.ACT_RELU, "gelu_tanh": L.ACT_GELU_TANH, "silu": L.ACT_SILU}


class TokenLogprobs(typing.NamedTuple):
    """Of every row: the target's log probability, the entropy (fp32 [n]), the
    statistics the backward pass takes (fp32 [n, 2]) and the likeliest tokens with
    their log probabilities ([n, top] int64 and fp32; None where top is 0)."""
    logprob: torch.Tensor
    entropy: torch.Tensor
    stats: torch.Tensor
    top_logprobs: torch.Tensor | None
    top_ids: torch.Tensor | None


def _check(rc: int):
    if rc != L.OK:
        raise MLKVError(rc, L.load().mlkv_status_string(rc).decode())


def _matrix(x, name: str, dtypes=_TYPES, shape=None, device=None) -> torch.Tensor:
    """The tensor, with contiguous rows that do not overlap."""
    try:
        rows, cols = x.shape
        dtype = x.dtype
    except (AttributeError, ValueError):
        raise TypeError(f"{name} must be a 2-d tensor") from None
    if dtype not in (dtypes or _TYPES):
        raise TypeError(f"{name} must be of {' or '.join(str(d) for d in dtypes or _TYPES)}, not {dtype}")
    if device is not None and x.device != device:
        raise TypeError(f"{name} must be on {device}, not {x.device}")
    if shape is not None and (rows, cols) != shape:
        raise ValueError(f"{name} must be {list(shape)}, not {list(x.shape)}")
    along, across = x.stride()
    if across != 1 and cols > 1 or along < cols and rows > 1:
        return x.contiguous()
    return x


def _row_stride(x: torch.Tensor) -> int:
    rows, cols = x.shape
    return x.stride(0) if rows > 1 else cols


def _vector(x, name: str, n: int, device, dtypes) -> torch.Tensor:
    if not isinstance(x, torch.Tensor) or x.dim() != 1 or x.dtype not in dtypes or x.device != device:
        raise TypeError(f"{name} must be a 1-d tensor of {' or '.join(str(d) for d in dtypes)} on {device}")
    if x.shape[0] != n:
        raise ValueError(f"{name} must have {n} values, not {x.shape[0]}")
    return x if x.is_contiguous() else x.contiguous()


def _on_gpu(x: torch.Tensor, name: str):
    if not x.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")


_HERE = contextlib.nullcontext()


def _current(device):
    """Makes the device current for a library call (nothing to do, as a rule)."""
    return _HERE if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _ptr(x) -> int | None:
    return None if x is None else x.data_ptr()


def _workspace(size: int, device):
    if size < 0:
        raise MLKVError(L.ERR_INVALID, "sizes that the operator does not take")
    return torch.empty(size, dtype=torch.uint8, device=device) if size else None


# -- layer norm ------------------------------------------------------------------
def _norm_weights(weight, bias, dim, device):
    types = tuple(_TYPES) if weight is None else (weight.dtype,)
    w = None if weight is None else _vector(weight, "weight", dim, device, tuple(_TYPES))
    b = None if bias is None else _vector(bias, "bias", dim, device, types)
    kind = _TYPES[w.dtype] if w is not None else _TYPES[b.dtype] if b is not None else L.TYPE_FLOAT
    return w, b, kind


def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, *,
               eps: float = 1e-5, out_dtype: torch.dtype | None = None, save_stats: bool = False):
    """(x - mean) / sqrt(var + eps) * weight + bias, row by row: [rows, dim] of
    out_dtype (x's; any type where x is fp32).  weight and bias: [dim], of one type.
    With save_stats also the rows' (mean, 1 / sqrt(var + eps)), fp32 [rows, 2], for
    layer_norm_backward."""
    x = _matrix(x, "x")
    _on_gpu(x, "x")
    rows, dim = x.shape
    out_dtype = x.dtype if out_dtype is None else out_dtype
    if out_dtype not in _TYPES or x.dtype != torch.float32 and out_dtype != x.dtype:
        raise TypeError(f"out_dtype {out_dtype} of x's {x.dtype}")
    w, b, kind = _norm_weights(weight, bias, dim, x.device)
    y = torch.empty((rows, dim), dtype=out_dtype, device=x.device)
    stats = torch.empty((rows, 2), dtype=torch.float32, device=x.device) if save_stats else None
    with _current(x.device):
        _check(L.load().mlkv_layer_norm(x.data_ptr(), _row_stride(x), _TYPES[x.dtype], rows, dim, _ptr(w), _ptr(b), kind,
                                        eps, y.data_ptr(), dim, _TYPES[out_dtype], _ptr(stats), _stream(x.device)))
    return (y, stats) if save_stats else y


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor | None, stats: torch.Tensor, *,
                        bias: bool = True):
    """Gradients (dx of x's type, dweight, dbias of the weight's type or fp32) of a
    layer_norm whose save_stats gave `stats`; dweight is None without a weight, dbias
    with bias=False."""
    x = _matrix(x, "x")
    _on_gpu(x, "x")
    rows, dim = x.shape
    dy = _matrix(dy, "dy", tuple(_TYPES) if x.dtype == torch.float32 else (x.dtype,), (rows, dim), x.device)
    stats = _matrix(stats, "stats", (torch.float32,), (rows, 2), x.device).contiguous()
    w, _, kind = _norm_weights(weight, None, dim, x.device)
    dx = torch.empty((rows, dim), dtype=x.dtype, device=x.device)
    wt = torch.float32 if w is None else w.dtype
    dw = None if w is None else torch.empty(dim, dtype=wt, device=x.device)
    db = torch.empty(dim, dtype=wt, device=x.device) if bias else None
    lib = L.load()
    with _current(x.device):
        size = lib.mlkv_layer_norm_backward_workspace(rows, dim)
        ws = _workspace(size, x.device)
        _check(lib.mlkv_layer_norm_backward(dy.data_ptr(), _row_stride(dy), _TYPES[dy.dtype], x.data_ptr(), _row_stride(x),
                                            _TYPES[x.dtype], rows, dim, _ptr(w), kind, stats.data_ptr(), dx.data_ptr(), dim,
                                            _ptr(dw), _ptr(db), _ptr(ws), size,
                                            _stream(x.device)))
    return dx, dw, db


# -- matrix products ----------------------------------------------------------------
_HALVES = (torch.bfloat16, torch.float16)


def _linear_args(x, weight, activation):
    """(x, weight, their device, the call's arguments so far)"""
    x = _matrix(x, "x", _HALVES)
    _on_gpu(x, "x")
    m, k = x.shape
    dtype, device = x.dtype, x.device
    weight = _matrix(weight, "weight", (dtype,), None, device)
    n, along = weight.shape
    if along != k:
        raise ValueError(f"weight must be [n, {k}], not {list(weight.shape)}")
    act = _ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {', '.join(filter(None, _ACTIVATIONS))}, not {activation!r}")
    return x, weight, device, L.LinearArgs(m=m, n=n, k=k, d_x=x.data_ptr(), x_stride=_row_stride(x), d_weight=weight.data_ptr(),
                                           weight_stride=_row_stride(weight), type=_TYPES[dtype], activation=act)


def _run_linear(call, workspace, args, device):
    with _current(device):
        size = workspace(args)
        if size:
            ws = _workspace(size, device)
            args.d_workspace, args.workspace_bytes = ws.data_ptr(), size
        _check(call(args, _stream(device)))


def linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, *, activation: str | None = None,
           residual: torch.Tensor | None = None, save_pre: bool = False):
    """act(x @ weight.T + bias) + residual: x [m, k], weight [n, k], bias [n], residual
    [m, n], all of x's type; activation: "none", "relu", "gelu_tanh" or "silu".  With
    save_pre also the value before the activation, [m, n], for linear_backward (None
    without an activation, whose gradient does not need it)."""
    x, weight, device, a = _linear_args(x, weight, activation)
    m, n, dtype = a.m, a.n, x.dtype
    if bias is not None:
        bias = _vector(bias, "bias", n, device, (dtype,))
        a.d_bias = bias.data_ptr()
    if residual is not None:
        residual = _matrix(residual, "residual", (dtype,), (m, n), device)
        a.d_residual, a.residual_stride = residual.data_ptr(), _row_stride(residual)
    y = torch.empty((m, n), dtype=dtype, device=device)
    a.d_y, a.y_stride = y.data_ptr(), n
    pre = None
    if save_pre and a.activation != L.ACT_NONE:
        pre = torch.empty((m, n), dtype=dtype, device=device)
        a.d_pre, a.pre_stride = pre.data_ptr(), n
    lib = L.load()
    _run_linear(lib.mlkv_linear, lib.mlkv_linear_workspace, a, device)
    return (y, pre) if save_pre else y


def linear_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, pre: torch.Tensor | None = None, *,
                    activation: str | None = None, bias: bool = False, want_dx: bool = True, want_dweight: bool = True):
    """Gradients (dx, dweight, dbias) of linear(x, weight, bias, activation=...), all of
    x's type; dbias is None without `bias`, the others where they are not wanted.  pre:
    what save_pre gave (needed with an activation).  The residual's gradient is dy."""
    x, weight, device, a = _linear_args(x, weight, activation)
    m, n, k, dtype = a.m, a.n, a.k, x.dtype
    dy = _matrix(dy, "dy", (dtype,), (m, n), device)
    a.d_dy, a.dy_stride = dy.data_ptr(), _row_stride(dy)
    if a.activation != L.ACT_NONE:
        if pre is None:
            raise TypeError("pre is needed for the gradient of an activation")
        pre = _matrix(pre, "pre", (dtype,), (m, n), device)
        a.d_pre, a.pre_stride = pre.data_ptr(), _row_stride(pre)
    dx = dw = db = None
    if want_dx:
        dx = torch.empty((m, k), dtype=dtype, device=device)
        a.d_dx, a.dx_stride = dx.data_ptr(), k
    if want_dweight:
        dw = torch.empty((n, k), dtype=dtype, device=device)
        a.d_dweight, a.dweight_stride = dw.data_ptr(), k
    if bias:
        db = torch.empty(n, dtype=dtype, device=device)
        a.d_dbias = db.data_ptr()
    lib = L.load()
    _run_linear(lib.mlkv_linear_backward, lib.mlkv_linear_backward_workspace, a, device)
    return dx, dw, db


def sync(device=None):
    """Waits for the current stream; raises if a bounded wait inside a product's kernel
    ran out since the last call (its outputs are then not valid)."""
    device = torch.device("cuda", torch.cuda.current_device() if device is None else torch.device(device).index or 0)
    with torch.cuda.device(device):
        _check(L.load().mlkv_dense_sync(_stream(device)))


# -- log probabilities ------------------------------------------------------------------
def _logits(logits, targets, scale):
    logits = _matrix(logits, "logits")
    _on_gpu(logits, "logits")
    if logits.shape[1] < 1:
        raise ValueError("logits must have at least one column")
    if not 0 < scale < float("inf"):
        raise ValueError(f"scale must be positive and finite, not {scale}")
    return logits, _vector(targets, "targets", logits.shape[0], logits.device, (torch.int64,))


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, *, top: int = 0, scale: float = 1.0) -> TokenLogprobs:
    """Of every row of softmax(scale * logits) ([n, vocab]): the log probability of
    targets[i] (int64 [n]; negative: none, log probability 0), the entropy, and the
    `top` (at most 32) likeliest tokens, ties by the lowest index.  -inf masks a token."""
    logits, targets = _logits(logits, targets, scale)
    if not 0 <= top <= L.MAX_TOP:
        raise ValueError(f"top must be 0 to {L.MAX_TOP}, not {top}")
    n, vocab = logits.shape
    dev = logits.device
    logprob = torch.empty(n, dtype=torch.float32, device=dev)
    entropy = torch.empty(n, dtype=torch.float32, device=dev)
    stats = torch.empty((n, 2), dtype=torch.float32, device=dev)
    tops = torch.empty((n, top), dtype=torch.float32, device=dev) if top else None
    ids = torch.empty((n, top), dtype=torch.int64, device=dev) if top else None
    lib = L.load()
    kind = _TYPES[logits.dtype]
    with _current(dev):
        size = lib.mlkv_token_logprobs_workspace(n, vocab, kind, top)
        ws = _workspace(size, dev) if size else None
        _check(lib.mlkv_token_logprobs(logits.data_ptr(), _row_stride(logits), kind, n, vocab, targets.data_ptr(), scale,
                                       top, logprob.data_ptr(), entropy.data_ptr(), stats.data_ptr(), _ptr(tops),
                                       _ptr(ids), _ptr(ws), size, _stream(dev)))
    return TokenLogprobs(logprob, entropy, stats, tops, ids)


def token_logprobs_backward(logits: torch.Tensor, targets: torch.Tensor, result: TokenLogprobs,
                            dlogprob: torch.Tensor | None = None, dentropy: torch.Tensor | None = None, *,
                            scale: float = 1.0, in_place: bool = False) -> torch.Tensor:
    """The gradient of the logits, of their type, from those of the log probabilities
    and entropies (fp32 [n]; None: 0) that token_logprobs of the same arguments gave in
    `result`.  in_place: written over the logits."""
    given = logits
    logits, targets = _logits(logits, targets, scale)
    n, vocab = logits.shape
    dev = logits.device
    stats = _matrix(result.stats, "result.stats", (torch.float32,), (n, 2), dev).contiguous()
    entropy = _vector(result.entropy, "result.entropy", n, dev, (torch.float32,))
    g = None if dlogprob is None else _vector(dlogprob, "dlogprob", n, dev, (torch.float32,))
    h = None if dentropy is None else _vector(dentropy, "dentropy", n, dev, (torch.float32,))
    if in_place and logits is not given:
        raise TypeError("logits written in place must have contiguous rows")
    out = logits if in_place else torch.empty((n, vocab), dtype=logits.dtype, device=dev)
    with _current(dev):
        _check(L.load().mlkv_token_logprobs_backward(logits.data_ptr(), _row_stride(logits), _TYPES[logits.dtype], n, vocab,
                                                     targets.data_ptr(), scale, entropy.data_ptr(), stats.data_ptr(),
                                                     _ptr(g), _ptr(h), out.data_ptr(), _row_stride(out), _stream(dev)))
    return out
