"""The dense operators' definitions in 64 bits, and how far 32-bit sums and one
rounding to the output's type may lie from them, element by element.

Bounds: a sum of n products in fp32, in any order and rounded or cut at every
step, is off by at most (n + 8) 2^-23 of the sum of their magnitudes; a value
rounded to a type with p bits is off by 2^-p of itself (and, for fp16, 2^-25).
exp, division and root add a few units of 2^-22, which the constants below hold.
"""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
F32 = 2.0 ** -23


def rounding(v, dtype):
    return UNIT[dtype] * v.abs() + LEAST[dtype]


def within(got, want, tol, what=""):
    """got (any type) within tol of want, element by element; not finite where want is not."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    g, w = got.double(), want.double()
    same = (g == w) | (g.isnan() & w.isnan())
    err = torch.where(same, torch.zeros_like(w), (g - w).abs())
    bad = ~same & ~(err <= tol)
    if bad.any():
        i = (err / tol.clamp(min=1e-300)).nan_to_num(math.inf).where(bad, torch.zeros_like(err)).argmax()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; worst at {int(i)}: "
                             f"{g.flatten()[i].item()} for {w.flatten()[i].item()}, tolerance {tol.expand_as(w).flatten()[i].item()}")


# -- layer norm ---------------------------------------------------------------------
def layer_norm(x, w, b, eps):
    """(y, tolerance of y before its rounding, mean, rstd)."""
    x = x.double()
    dim = x.shape[1]
    w = torch.ones(dim, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(dim, dtype=torch.float64, device=x.device) if b is None else b.double()
    mu = x.mean(1, keepdim=True)
    var = ((x - mu) ** 2).mean(1, keepdim=True)
    r = 1 / torch.sqrt(var + eps)
    xh = (x - mu) * r
    # chains of at most 64 additions a lane, 5 shuffles, 32 warps
    n = min(dim, 64) + 40
    dmu = n * F32 * x.abs().mean(1, keepdim=True)
    d = x - mu
    # the variance about a mean off by dmu is off by dmu^2, its root's relative error by half of the variance's
    rel = n * F32 + dmu ** 2 * r ** 2 + (dmu + F32 * d.abs().mean(1, keepdim=True)) * r * 2 ** -10 + 4 * F32
    tol = (dmu + F32 * d.abs()) * r * w.abs() + (rel + 4 * F32) * (xh * w).abs() + F32 * (b.abs() + (xh * w + b).abs())
    return xh * w + b, tol, mu, r, xh, rel, dmu


def layer_norm_backward(dy, x, w, eps):
    """(dx, dw, db) with their tolerances."""
    _, _, mu, r, xh, rel, dmu = layer_norm(x, w, None, eps)
    rows, dim = x.shape
    dy = dy.double()
    w = torch.ones(dim, dtype=torch.float64, device=x.device) if w is None else w.double()
    g = dy * w
    c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = r * (g - c1 - xh * c2)
    n = min(dim, 64) + 40
    dxh = dmu * r + (rel + 4 * F32) * xh.abs()                   # error of xh
    dc1 = n * F32 * g.abs().mean(1, keepdim=True)
    dc2 = n * F32 * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * dxh).mean(1, keepdim=True)
    tol = r * (dc1 + xh.abs() * dc2 + dxh * c2.abs() + 4 * F32 * (g.abs() + c1.abs() + (xh * c2).abs())) + (rel + 4 * F32) * dx.abs()
    dw, db = (dy * xh).sum(0), dy.sum(0)
    tw = (rows + 8) * F32 * (dy * xh).abs().sum(0) + (dy.abs() * dxh).sum(0)
    tb = (rows + 8) * F32 * dy.abs().sum(0)
    return (dx, tol), (dw, tw), (db, tb)


# -- matrix products -----------------------------------------------------------------
def act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def act_slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "silu":
        q = torch.sigmoid(z)
        return q * (1 + z * (1 - q))
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


SLOPE = 1.13     # most of any activation's slope ...
BEND = 1.2       # ... and of any slope's slope (relu's step apart)


def linear(x, w, b, name, res):
    """(y, tolerance before its rounding, z, tolerance of z)."""
    x, w = x.double(), w.double()
    k = x.shape[1]
    z = x @ w.T
    tz = (k + 8) * F32 * (x.abs() @ w.abs().T)
    if b is not None:
        z = z + b.double()
        tz = tz + F32 * z.abs()
    y = act(z, name)
    ty = SLOPE * tz + (0 if name == "none" else 2.0 ** -18 * y.abs() + 2.0 ** -126)
    if res is not None:
        y = y + res.double()
        ty = ty + F32 * y.abs()
    return y, ty, z, tz


def linear_backward(dy, x, w, b, name, dtype):
    """(dx, dw, db) with their tolerances before rounding."""
    _, _, z, tz = linear(x, w, b, name, None)
    dy, x, w = dy.double(), x.double(), w.double()
    p = dy * act_slope(z, name)
    if name == "none":
        tp = torch.zeros_like(p)
    else:
        dz = tz + rounding(z.abs() + tz, dtype)                   # of the saved value
        if name == "relu":
            tp = torch.where(z.abs() <= dz, dy.abs(), torch.zeros_like(p)) + rounding(p, dtype)
        else:
            tp = dy.abs() * BEND * dz + 2.0 ** -18 * p.abs() + rounding(p, dtype) * 1.01
    m, n = dy.shape
    a = p.abs() + tp
    dx, tx = p @ w, tp @ w.abs() + (n + 8) * F32 * (a @ w.abs())
    dw, tw = p.T @ x, tp.T @ x.abs() + (m + 8) * F32 * (a.T @ x.abs())
    db, tb = p.sum(0), tp.sum(0) + (m + 8) * F32 * a.sum(0)
    return (dx, tx), (dw, tw), (db, tb)


# -- log probabilities ----------------------------------------------------------------
def token_logprobs(logits, targets, scale):
    """(logprob, entropy, log probabilities of all, rows without a token)."""
    x = logits.double()
    top = x.amax(1, keepdim=True)
    empty = (x == -math.inf).all(1)
    d = (x - torch.where(empty[:, None], torch.zeros_like(top), top)) * scale
    logs = torch.log(torch.exp(d).sum(1, keepdim=True))
    lp = d - logs
    lp[empty] = -math.inf
    ent = -torch.where(torch.exp(lp) > 0, torch.exp(lp) * lp, torch.zeros_like(lp)).sum(1)
    bad = (x.isnan() | (x == math.inf)).any(1)
    lp[bad], ent[bad] = math.nan, math.nan
    tok = lp.gather(1, targets.clamp(0, x.shape[1] - 1)[:, None])[:, 0]
    tok = torch.where(targets >= x.shape[1], torch.full_like(tok, math.nan), tok)
    tok = torch.where(targets < 0, torch.zeros_like(tok), tok)
    return tok, ent, lp, empty


def alternatives(logits, top):
    """Ids by falling value, then rising index (NaN first); -1 for -inf and what is left over."""
    x = logits.double() + 0.0
    n, v = x.shape
    order = torch.where(x.isnan(), torch.full_like(x, math.inf), x)
    # stable sorts, the last the most significant: value, then NaN before +inf
    ids = order.sort(dim=1, descending=True, stable=True).indices
    nan = x.gather(1, ids).isnan()
    ids = ids.gather(1, nan.to(torch.int8).sort(dim=1, descending=True, stable=True).indices)
    ids = torch.where(x.gather(1, ids) == -math.inf, -1, ids)[:, :top]
    return torch.nn.functional.pad(ids, (0, top - ids.shape[1]), value=-1)


def token_logprobs_backward(logits, targets, scale, g, h):
    """(dlogits, tolerance before rounding)."""
    x = logits.double()
    n, v = x.shape
    _, ent, lp, empty = token_logprobs(logits, targets, scale)
    g = torch.zeros(n, dtype=torch.float64, device=x.device) if g is None else g.double()
    h = torch.zeros(n, dtype=torch.float64, device=x.device) if h is None else h.double()
    g = torch.where(targets < 0, torch.zeros_like(g), g)[:, None]
    h = h[:, None]
    p = torch.exp(lp)
    l0 = torch.where(p > 0, lp, torch.zeros_like(lp))
    e0 = ent[:, None]
    dz = -p * (g + h * (l0 + e0))
    mag = p * (g.abs() + h.abs() * (l0.abs() + e0 + 1)) * (1 + l0.abs())
    at = torch.zeros_like(x, dtype=torch.bool).scatter_(1, targets.clamp(0, v - 1)[:, None], True)
    dz = torch.where(at, dz + g, dz)
    mag = torch.where(at, mag + g.abs(), mag)
    dz = torch.where(x == -math.inf, torch.zeros_like(dz), dz)
    bad = targets >= v
    dz[bad], mag[bad] = math.nan, 0.0
    return dz * scale, 2.0 ** -16 * scale * mag + 2.0 ** -100
