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
only checks arguments (TypeError, ValueError) and passes pointers; where nothing
is wrong with them and nothing has to be copied, _dense_calls does (csrc/dense_calls.cpp:
the host's part of a call is what a small one takes; without that module this one
makes every call).  Formulas, the treatment of masked and invalid values, and what
takes longer for the data's sake: include/mlkv_dense.h.

Nothing here is recorded for torch's autograd, whether or not an argument requires
a gradient: what a call returns has no history, and the gradients are what the
*_backward calls return.
"""
import typing
import warnings

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


_calls = None


def _native(x):
    """The calls for arguments as the library takes them, where x is a CUDA tensor."""
    global _calls
    if not getattr(x, "is_cuda", False):
        return None
    if _calls is None:
        lib = L.load()
        try:
            from . import _dense_calls
        except ImportError as e:
            warnings.warn(f"the dense operators' extension module is missing, calls take 10 us or so longer: build it with "
                          f"__graft_entry__.build() ({e})", RuntimeWarning, stacklevel=3)
            _calls = ()
        else:
            _dense_calls.bind(lib._name)
            _calls = _dense_calls
    return _calls or None


def _done(result):
    """What a call of _native's gave, or the error that it tells."""
    if type(result) is int:
        raise MLKVError(result, L.load().mlkv_status_string(result).decode())
    return result


_current_device = torch.cuda.current_device
_empty = torch.empty


def _call(device, call, *args):
    """call(*args) with the device current (which it is, as a rule)."""
    if _current_device() == device.index:
        rc = call(*args)
    else:
        with torch.cuda.device(device):
            rc = call(*args)
    if rc != L.OK:
        raise MLKVError(rc, L.load().mlkv_status_string(rc).decode())


def _names(dtypes) -> str:
    return " or ".join(str(d) for d in dtypes)


def _rows(x, name: str, dtypes=_TYPES, shape=None, device=None):
    """(the tensor, with contiguous rows that do not overlap; rows; columns; row stride)"""
    try:
        rows, cols = x.shape
        along, across = x.stride()
        dtype = x.dtype
    except (AttributeError, ValueError):
        raise TypeError(f"{name} must be a 2-d tensor") from None
    if dtype not in dtypes:
        raise TypeError(f"{name} must be of {_names(dtypes)}, not {dtype}")
    if device is not None and x.device != device:
        raise TypeError(f"{name} must be on {device}, not {x.device}")
    if shape is not None and (rows, cols) != shape:
        raise ValueError(f"{name} must be {list(shape)}, not {[rows, cols]}")
    if across != 1 and cols > 1 or along < cols and rows > 1:
        return x.contiguous(), rows, cols, cols
    return x, rows, cols, along if rows > 1 else cols


def _matrix(x, name: str, dtypes=None, shape=None, device=None) -> torch.Tensor:
    return _rows(x, name, dtypes or _TYPES, shape, device)[0]


def _row_stride(x: torch.Tensor) -> int:
    return _rows(x, "x")[3]


def _vector(x, name: str, n: int, device, dtypes) -> torch.Tensor:
    try:
        (size,) = x.shape
        (step,) = x.stride()
        fits = x.dtype in dtypes and x.device == device
    except (AttributeError, ValueError):
        fits = False
    if not fits:
        raise TypeError(f"{name} must be a 1-d tensor of {_names(dtypes)} on {device}")
    if size != n:
        raise ValueError(f"{name} must have {n} values, not {size}")
    return x if step == 1 else x.contiguous()


def _on_gpu(x: torch.Tensor, name: str):
    if not x.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")


def _workspace(size: int, device):
    """(a tensor to keep until the call is made, its address) for so many bytes."""
    if size <= 0:
        if size < 0:
            raise MLKVError(L.ERR_INVALID, "sizes that the operator does not take")
        return None, None
    ws = _empty(size, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr()


# -- layer norm ------------------------------------------------------------------
def layer_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, *,
               eps: float = 1e-5, out_dtype: torch.dtype | None = None, save_stats: bool = False):
    """(x - mean) / sqrt(var + eps) * weight + bias, row by row: [rows, dim] of
    out_dtype (x's; any type where x is fp32).  weight and bias: [dim], of one type.
    With save_stats also the rows' (mean, 1 / sqrt(var + eps)), fp32 [rows, 2], for
    layer_norm_backward."""
    if (native := _native(x)) is not None:
        r = native.layer_norm(x, weight, bias, eps, -1 if out_dtype is None else _TYPES.get(out_dtype, -2), save_stats)
        if r is not NotImplemented:
            return _done(r)
    x, rows, dim, stride = _rows(x, "x")
    _on_gpu(x, "x")
    dtype, device = x.dtype, x.device
    if out_dtype is None:
        out_dtype = dtype
    elif out_dtype != dtype and (out_dtype not in _TYPES or dtype != torch.float32):
        raise TypeError(f"out_dtype {out_dtype} of x's {dtype}")
    w = b = None
    kind = L.TYPE_FLOAT
    if weight is not None:
        weight = _vector(weight, "weight", dim, device, _TYPES)
        w, kind = weight.data_ptr(), _TYPES[weight.dtype]
    if bias is not None:
        bias = _vector(bias, "bias", dim, device, _TYPES if weight is None else (weight.dtype,))
        b, kind = bias.data_ptr(), _TYPES[bias.dtype]
    y = _empty((rows, dim), dtype=out_dtype, device=device)
    stats = _empty((rows, 2), dtype=torch.float32, device=device) if save_stats else None
    _call(device, L.load().mlkv_layer_norm, x.data_ptr(), stride, _TYPES[dtype], rows, dim, w, b, kind, eps, y.data_ptr(), dim,
          _TYPES[out_dtype], stats.data_ptr() if save_stats else None, _stream(device))
    return (y, stats) if save_stats else y


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor | None, stats: torch.Tensor, *,
                        bias: bool = True):
    """Gradients (dx of x's type, dweight, dbias of the weight's type or fp32) of a
    layer_norm whose save_stats gave `stats`; dweight is None without a weight, dbias
    with bias=False."""
    if (native := _native(x)) is not None:
        r = native.layer_norm_backward(dy, x, weight, stats, bias)
        if r is not NotImplemented:
            return _done(r)
    x, rows, dim, stride = _rows(x, "x")
    _on_gpu(x, "x")
    dtype, device = x.dtype, x.device
    dy, _, _, dy_stride = _rows(dy, "dy", _TYPES if dtype == torch.float32 else (dtype,), (rows, dim), device)
    stats = _rows(stats, "stats", (torch.float32,), (rows, 2), device)[0].contiguous()
    dx = _empty((rows, dim), dtype=dtype, device=device)
    dw = db = w = wt = None
    if weight is not None:
        weight = _vector(weight, "weight", dim, device, _TYPES)
        w, wt = weight.data_ptr(), weight.dtype
        dw = _empty(dim, dtype=wt, device=device)
    else:
        wt = torch.float32
    if bias:
        db = _empty(dim, dtype=wt, device=device)
    lib = L.load()
    size = lib.mlkv_layer_norm_backward_workspace(rows, dim)
    ws, at = _workspace(size, device)
    _call(device, lib.mlkv_layer_norm_backward, dy.data_ptr(), dy_stride, _TYPES[dy.dtype], x.data_ptr(), stride, _TYPES[dtype],
          rows, dim, w, _TYPES[wt], stats.data_ptr(), dx.data_ptr(), dim, dw.data_ptr() if w is not None else None,
          db.data_ptr() if bias else None, at, size, _stream(device))
    return dx, dw, db


# -- matrix products ----------------------------------------------------------------
_HALVES = (torch.bfloat16, torch.float16)


def _linear_args(x, weight, activation):
    """(x, weight, their device, the call's arguments so far)"""
    x, m, k, x_stride = _rows(x, "x", _HALVES)
    _on_gpu(x, "x")
    dtype, device = x.dtype, x.device
    weight, n, along, weight_stride = _rows(weight, "weight", (dtype,), None, device)
    if along != k:
        raise ValueError(f"weight must be [n, {k}], not {[n, along]}")
    act = _ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {', '.join(filter(None, _ACTIVATIONS))}, not {activation!r}")
    a = L.LinearArgs(m, n, k, x.data_ptr(), x_stride, weight.data_ptr(), weight_stride)
    a.type = _TYPES[dtype]
    a.activation = act
    return x, weight, dtype, device, m, n, k, act, a


def _run_linear(call, workspace, args, device):
    size = workspace(args)
    if size:
        ws, args.d_workspace = _workspace(size, device)
        args.workspace_bytes = size
    _call(device, call, args, _stream(device))


def linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, *, activation: str | None = None,
           residual: torch.Tensor | None = None, save_pre: bool = False):
    """act(x @ weight.T + bias) + residual: x [m, k], weight [n, k], bias [n], residual
    [m, n], all of x's type; activation: "none", "relu", "gelu_tanh" or "silu".  With
    save_pre also the value before the activation, [m, n], rounded to x's type, for
    linear_backward (None without an activation, whose gradient does not need it).  That the kernel's waits
    were all met, and the outputs are valid, is known after sync()."""
    if (native := _native(x)) is not None:
        r = native.linear(x, weight, bias, _ACTIVATIONS.get(activation, -1), residual, save_pre)
        if r is not NotImplemented:
            return _done(r)
    x, weight, dtype, device, m, n, k, act, a = _linear_args(x, weight, activation)
    if bias is not None:
        bias = _vector(bias, "bias", n, device, (dtype,))
        a.d_bias = bias.data_ptr()
    if residual is not None:
        residual, _, _, a.residual_stride = _rows(residual, "residual", (dtype,), (m, n), device)
        a.d_residual = residual.data_ptr()
    y = _empty((m, n), dtype=dtype, device=device)
    a.d_y, a.y_stride = y.data_ptr(), n
    pre = None
    if save_pre and act != L.ACT_NONE:
        pre = _empty((m, n), dtype=dtype, device=device)
        a.d_pre, a.pre_stride = pre.data_ptr(), n
    lib = L.load()
    _run_linear(lib.mlkv_linear, lib.mlkv_linear_workspace, a, device)
    return (y, pre) if save_pre else y


def linear_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, pre: torch.Tensor | None = None, *,
                    activation: str | None = None, bias: bool = False, want_dx: bool = True, want_dweight: bool = True):
    """Gradients (dx, dweight, dbias) of linear(x, weight, bias, activation=...), all of
    x's type; dbias is None without `bias`, the others where they are not wanted.  pre:
    what save_pre gave (needed with an activation): the slopes are taken there, and dy
    times them is rounded to x's type.  The residual's gradient is dy.
    Valid when sync() says so, as linear's."""
    if (native := _native(x)) is not None:
        r = native.linear_backward(dy, x, weight, pre, _ACTIVATIONS.get(activation, -1), bias, want_dx, want_dweight)
        if r is not NotImplemented:
            return _done(r)
    x, weight, dtype, device, m, n, k, act, a = _linear_args(x, weight, activation)
    dy, _, _, a.dy_stride = _rows(dy, "dy", (dtype,), (m, n), device)
    a.d_dy = dy.data_ptr()
    if act != L.ACT_NONE:
        if pre is None:
            raise TypeError("pre is needed for the gradient of an activation")
        pre, _, _, a.pre_stride = _rows(pre, "pre", (dtype,), (m, n), device)
        a.d_pre = pre.data_ptr()
    dx = dw = db = None
    if want_dx:
        dx = _empty((m, k), dtype=dtype, device=device)
        a.d_dx, a.dx_stride = dx.data_ptr(), k
    if want_dweight:
        dw = _empty((n, k), dtype=dtype, device=device)
        a.d_dweight, a.dweight_stride = dw.data_ptr(), k
    if bias:
        db = _empty(n, dtype=dtype, device=device)
        a.d_dbias = db.data_ptr()
    lib = L.load()
    _run_linear(lib.mlkv_linear_backward, lib.mlkv_linear_backward_workspace, a, device)
    return dx, dw, db


def sync(device=None):
    """Waits for the current stream; raises if a bounded wait inside a product's kernel
    ran out on the device, on any stream, since a call last raised for one (the
    outputs of that product are then not valid)."""
    device = torch.device("cuda" if device is None else device)
    if device.type != "cuda":
        raise TypeError(f"device must be a CUDA device, not {device}")
    if device.index is None:
        device = torch.device("cuda", _current_device())
    _call(device, L.load().mlkv_dense_sync, _stream(device))


# -- log probabilities ------------------------------------------------------------------
def _logits(logits, targets, scale):
    logits, n, vocab, stride = _rows(logits, "logits")
    _on_gpu(logits, "logits")
    if vocab < 1:
        raise ValueError("logits must have at least one column")
    if not 0 < scale < float("inf"):
        raise ValueError(f"scale must be positive and finite, not {scale}")
    device = logits.device
    return logits, n, vocab, stride, device, _vector(targets, "targets", n, device, (torch.int64,))


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, *, top: int = 0, scale: float = 1.0) -> TokenLogprobs:
    """Of every row of softmax(scale * logits) ([n, vocab]): the log probability of
    targets[i] (int64 [n]; negative: none, log probability 0), the entropy, and the
    `top` (at most 32) likeliest tokens, ties by the lowest index.  -inf masks a token."""
    if (native := _native(logits)) is not None:
        r = native.token_logprobs(logits, targets, top, scale)
        if r is not NotImplemented:
            return TokenLogprobs(*_done(r))
    logits, n, vocab, stride, device, targets = _logits(logits, targets, scale)
    if not 0 <= top <= L.MAX_TOP:
        raise ValueError(f"top must be 0 to {L.MAX_TOP}, not {top}")
    f32 = torch.float32
    logprob = _empty(n, dtype=f32, device=device)
    entropy = _empty(n, dtype=f32, device=device)
    stats = _empty((n, 2), dtype=f32, device=device)
    tops = ids = tops_at = ids_at = None
    if top:
        tops = _empty((n, top), dtype=f32, device=device)
        ids = _empty((n, top), dtype=torch.int64, device=device)
        tops_at, ids_at = tops.data_ptr(), ids.data_ptr()
    lib = L.load()
    kind = _TYPES[logits.dtype]
    size = lib.mlkv_token_logprobs_workspace(n, vocab, kind, top)
    ws, at = _workspace(size, device)
    _call(device, lib.mlkv_token_logprobs, logits.data_ptr(), stride, kind, n, vocab, targets.data_ptr(), scale, top,
          logprob.data_ptr(), entropy.data_ptr(), stats.data_ptr(), tops_at, ids_at, at, size, _stream(device))
    return TokenLogprobs(logprob, entropy, stats, tops, ids)


def token_logprobs_backward(logits: torch.Tensor, targets: torch.Tensor, result: TokenLogprobs,
                            dlogprob: torch.Tensor | None = None, dentropy: torch.Tensor | None = None, *,
                            scale: float = 1.0, in_place: bool = False) -> torch.Tensor:
    """The gradient of the logits, of their type, from those of the log probabilities
    and entropies (fp32 [n]; None: 0) that token_logprobs of the same arguments gave in
    `result`.  in_place: written over the logits."""
    if (native := _native(logits)) is not None:
        r = native.token_logprobs_backward(logits, targets, result.entropy, result.stats, dlogprob, dentropy, scale, in_place)
        if r is not NotImplemented:
            return _done(r)
    given = logits
    logits, n, vocab, stride, device, targets = _logits(logits, targets, scale)
    f32 = (torch.float32,)
    stats = _rows(result.stats, "result.stats", f32, (n, 2), device)[0].contiguous()
    entropy = _vector(result.entropy, "result.entropy", n, device, f32)
    g = None if dlogprob is None else _vector(dlogprob, "dlogprob", n, device, f32)
    h = None if dentropy is None else _vector(dentropy, "dentropy", n, device, f32)
    if in_place:
        if logits is not given:
            raise TypeError("logits written in place must have contiguous rows")
        out, out_stride = logits, stride
    else:
        out, out_stride = _empty((n, vocab), dtype=logits.dtype, device=device), vocab
    _call(device, L.load().mlkv_token_logprobs_backward, logits.data_ptr(), stride, _TYPES[logits.dtype], n, vocab,
          targets.data_ptr(), scale, entropy.data_ptr(), stats.data_ptr(), None if g is None else g.data_ptr(),
          None if h is None else h.data_ptr(), out.data_ptr(), out_stride, _stream(device))
    return out
