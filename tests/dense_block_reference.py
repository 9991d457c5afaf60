"""The gated block and the cross entropy of a linear layer in 64 bits, and how far 32-bit sums and the roundings that
their headers state may lie from them, element by element (the bounds are dense_reference's)."""
import math

import torch

from dense_reference import BEND, F32, LEAST, SLOPE, UNIT, act, act_slope, rounding


def _product(x, w):
    """(x w^T, tolerance)"""
    return x @ w.T, (x.shape[1] + 8) * F32 * (x.abs() @ w.abs().T)


def gated(x, wg, wu, name, dtype):
    """(h, its tolerance with its rounding, (g, tolerance), (u, tolerance)), the last two before a rounding."""
    x, wg, wu = x.double(), wg.double(), wu.double()
    (g, tg), (u, tu) = _product(x, wg), _product(x, wu)
    a = act(g, name)
    ta = SLOPE * tg + (0 if name == "none" else 2.0 ** -18 * a.abs() + 2.0 ** -126)
    h = a * u
    t = ta * u.abs() + (a.abs() + ta) * tu + F32 * h.abs()
    return h, t + rounding(h.abs() + t, dtype), (g, tg), (u, tu)


def gated_backward(dh, x, wg, wu, name, dtype):
    """(dx, dw_gate, dw_up) with their tolerances before rounding."""
    _, _, (g, tg), (u, tu) = gated(x, wg, wu, name, dtype)
    dh, x, wg, wu = dh.double(), x.double(), wg.double(), wu.double()
    tg = tg + rounding(g.abs() + tg, dtype)  # of the saved values
    tu = tu + rounding(u.abs() + tu, dtype)
    s, a = act_slope(g, name), act(g, name)
    if name == "relu":
        ts = torch.where(g.abs() <= tg, torch.ones_like(g), torch.zeros_like(g))
    else:
        ts = BEND * tg if name != "none" else torch.zeros_like(g)
    ta = SLOPE * tg + (0 if name == "none" else 2.0 ** -18 * a.abs() + 2.0 ** -126)
    fast = 2.0 ** -18  # exp, the division and the products
    dg, du = dh * u * s, dh * a
    tdg = dh.abs() * (tu * (s.abs() + ts) + u.abs() * ts) + fast * (dg.abs() + dh.abs() * u.abs() * (name != "none" and name != "relu"))
    tdg = tdg + rounding(dg.abs() + tdg, dtype)
    tdu = dh.abs() * ta + fast * du.abs()
    tdu = tdu + rounding(du.abs() + tdu, dtype)
    m, f = dh.shape
    dx = dg @ wg + du @ wu
    tx = tdg @ wg.abs() + tdu @ wu.abs() + (2 * f + 8) * F32 * ((dg.abs() + tdg) @ wg.abs() + (du.abs() + tdu) @ wu.abs())
    out = [(dx, tx)]
    for d, t in ((dg, tdg), (du, tdu)):
        out.append((d.T @ x, t.T @ x.abs() + (m + 8) * F32 * ((d.abs() + t).T @ x.abs())))
    return out


def xent_rows(x, w, targets, scale):
    """(loss, its tolerance, z, log probabilities, the tolerance of a logit, of the log of the sum) of some rows."""
    x, w = x.double(), w.double()
    n, vocab = x.shape[0], w.shape[0]
    z, tz = _product(x, w)
    z, tz = z * scale, tz * scale + 2 * F32 * (z * scale).abs()
    lse = torch.logsumexp(z, 1)
    # exponents (differences from the largest, times the scale, rounded thrice), exp2, and sums of positive terms in
    # chains of at most a 64th of the vocabulary
    spread = (z.amax(1) - z.amin(1)).clamp(max=100)
    tl = tz.amax(1) + 4 * F32 * spread + 2.0 ** -20 + (vocab / 64 + 100) * F32
    at = targets.clamp(0, vocab - 1)[:, None]
    zt = z.gather(1, at)[:, 0]
    loss = torch.where(targets < 0, torch.zeros_like(lse), lse - zt)
    loss = torch.where(targets >= vocab, torch.full_like(loss, math.nan), loss)
    tol = torch.where(targets < 0, torch.zeros_like(lse), tl + tz.gather(1, at)[:, 0] + 4 * F32 * (lse.abs() + zt.abs() + z.amax(1).abs()))
    return loss, tol, z, z - lse[:, None], tz, tl


def xent_backward(dloss, x, w, targets, scale, dtype, rows=1 << 14):
    """((dx, tolerance), (dweight, tolerance)) before rounding, some rows at a time."""
    vocab, k = w.shape
    g = torch.where(targets < 0, torch.zeros_like(dloss), dloss).double() * scale
    least = 2 * LEAST[dtype] * float(g.abs().max()) / 2.0 ** 13 if g.numel() else 0.0  # (of the type, at the power of two that P is held in)
    wd = w.double()
    dx, tx, dw, tw = [], [], torch.zeros_like(wd), torch.zeros_like(wd)
    for a in range(0, x.shape[0], rows):
        xa, ta = x[a:a + rows].double(), targets[a:a + rows]
        _, _, z, lp, tz, tl = xent_rows(xa, w, ta, scale)
        ga = g[a:a + rows, None]
        p = torch.exp(lp)
        err = p * torch.expm1(tz + tl[:, None] + 4 * F32 * lp.abs().clamp(max=100) + 2.0 ** -19)
        hot = torch.zeros_like(p)
        some = (ta >= 0) & (ta < vocab)
        hot[some] = hot[some].scatter(1, ta[some][:, None], 1.0)
        q = ga * (p - hot)
        t = ga.abs() * (err + F32 * (p + hot))
        t = t + UNIT[dtype] * (q.abs() + t) + least
        dx.append(q @ wd)
        tx.append(t @ wd.abs() + (vocab + 8) * F32 * ((q.abs() + t) @ wd.abs()))
        dw += q.T @ xa
        tw += t.T @ xa.abs() + (x.shape[0] + 8) * F32 * ((q.abs() + t).T @ xa.abs())
    return (torch.cat(dx), torch.cat(tx)), (dw, tw)
