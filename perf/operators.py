"""The dense operators between a Get and the apply of its gradients, as they are measured.

Three operators, each alone: the layer norm of looked-up rows (with the gradients of its weight and bias), the
matrix product with bias, activation and residual (with its backward pass), and the log probabilities of given
tokens with entropy and the likeliest alternatives (with the gradient of the logits).  A "fwd" pass is serving's
or scoring's; a "step" pass is a training step's share of the operator: forward, then backward.

Dims 16 to 512, 100 among them, batches of 26 features a sample and 65,536 samples follow `workloads/configs.py`.
The widths of the dense network and of the vocabularies are generic: the workloads have none.

The plain form computes in 32 bits from elementary operations and rounds once at the end.  `exact` computes the
definitions in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


def _ln(rows, dim, x, y, w, step, pad=0):
    return dict(op="ln", rows=rows, dim=dim, x=x, y=y, w=w, step=step, pad=pad)


def _lin(m, k, n, t, act, bias, res, step, pad=0):
    return dict(op="linear", m=m, k=k, n=n, t=t, act=act, bias=bias, res=res, step=step, pad=pad)


def _lp(n, v, t, top, step, mask="none", scale=1.0, pad=0):
    return dict(op="logprobs", n=n, v=v, t=t, top=top, step=step, mask=mask, scale=scale, pad=pad)


def listed():
    return [
        # Serving: the looked-up features of 16 samples (26 tables), fp32 rows into 16 bits; nothing but latency.
        dict(name="ln_serve", **_ln(416, 128, "fp32", "bf16", "fp32", False)),
        # Training on knowledge-graph rows (dim 100: bf16 rows are no multiple of 16 bytes), an odd batch.
        dict(name="ln_kg_step", **_ln(200_003, 100, "fp32", "bf16", "fp32", True)),
        # Training a wide network: hidden 2,048 in bf16 throughout.
        dict(name="ln_wide_step", **_ln(65_536, 2_048, "bf16", "bf16", "bf16", True)),
        # A single token through a wide layer: the weight is read once, nothing else counts.
        dict(name="lin_token", **_lin(1, 4_096, 4_096, "bf16", "silu", True, True, False)),
        # A small serving batch through the up-projection of a two-layer block.
        dict(name="lin_serve", **_lin(26, 1_024, 4_096, "fp16", "gelu_tanh", True, False, False)),
        # An odd network on an odd batch: no row starts on a 16-byte boundary.
        dict(name="lin_odd_step", **_lin(4_099, 777, 1_001, "bf16", "relu", True, False, True)),
        # A recommendation tower's first layer: 65,536 samples, 26 features of dim 16 side by side.
        dict(name="lin_tower_step", **_lin(65_536, 416, 512, "bf16", "relu", True, False, True)),
        # Training a wide block: the largest product, all of the epilogue.
        dict(name="lin_wide_step", **_lin(16_384, 4_096, 4_096, "bf16", "gelu_tanh", True, True, True)),
        # One generated token: its log probability and 20 alternatives.
        dict(name="lp_token", **_lp(1, 131_072, "bf16", 20, False)),
        # Constrained scoring: a third of an odd vocabulary masked to -inf, some rows whole; a temperature.
        dict(name="lp_masked", **_lp(515, 50_001, "fp32", 5, False, mask="inf", scale=1.25)),
        # Training over relation-sized classes: 15,000 scores a sample, no alternatives.
        dict(name="lp_class_step", **_lp(16_384, 15_000, "fp16", 0, True)),
        # Policy training: the largest, 20 alternatives kept.
        dict(name="lp_wide_step", **_lp(8_192, 131_072, "bf16", 20, True)),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def _width(rng, lo, hi):
    """As _spread; mostly a multiple of 8, as widths are, else any."""
    v = _spread(rng, lo, hi)
    return v if rng.random() < 0.35 else max(lo, v // 8 * 8)


def draw(rng):
    """Rows 1 to 262,144 of dims 16 to 8,192; products of 1 to 16,384 rows over widths 16 to 8,192; 1 to 16,384 rows
    of 2 to 262,144 scores: every type, direction, activation and kind of mask, contiguous rows and slices of wider
    ones."""
    op = rng.choice(["ln", "linear", "linear", "logprobs"])
    step = rng.random() < 0.5
    pad = rng.choice([0, 0, 0, 8, 5])
    if op == "ln":
        dim = _width(rng, 16, 8_192)
        x = rng.choice(["fp32", "bf16", "fp16"])
        y = rng.choice(["bf16", "fp16", "fp32"]) if x == "fp32" else x
        return _ln(_spread(rng, 1, min(262_144, 65_536 * 2_048 // dim)), dim, x, y,
                   rng.choice(["fp32", x if x != "fp32" else "bf16"]), step, pad)
    if op == "linear":
        k, n = _width(rng, 16, 8_192), _width(rng, 16, 8_192)
        m = _spread(rng, 1, min(16_384, 16_384 * 4_096 * 4_096 // (n * k)))
        return _lin(m, k, n, rng.choice(["bf16", "fp16"]), rng.choice(["none", "relu", "gelu_tanh", "silu"]),
                    rng.random() < 0.7, rng.random() < 0.4, step, pad)
    v = _spread(rng, 2, 262_144) if rng.random() < 0.5 else _width(rng, 256, 262_144)
    t = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    most = 8_192 * 131_072 // (2 if t == "fp32" else 1)
    return _lp(_spread(rng, 1, min(16_384, most // v)), v, t, rng.choice([0, 1, 5, 20, 32]), step,
               rng.choice(["none", "none", "inf", "lowest" if v >= 256 else "none"]), rng.choice([1.0, 1.0, 0.7, 1.25]), pad)


# --- inputs -----------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator("cuda")
    g.manual_seed((seed * 1_000_003 + stream * 7_919 + 23) & 0x7FFF_FFFF_FFFF)
    return g


def _normal(shape, sigma, dtype, gen, mean=0.0, pad=0):
    """N(mean, sigma) values; with `pad`, rows that are slices of rows `pad` values wider."""
    full = (*shape[:-1], shape[-1] + pad)
    x = torch.empty(full, device="cuda", dtype=dtype).normal_(mean, sigma, generator=gen)
    return x[..., :shape[-1]] if pad else x


def prepare(case, seed):
    g = _gen(seed, 1)
    s = {"case": case}
    if case["op"] == "ln":
        rows, dim, xt, wt = case["rows"], case["dim"], TYPES[case["x"]], TYPES[case["w"]]
        x = _normal((rows, dim), 1.0, xt, g, mean=0.25, pad=case["pad"])
        x.mul_(_normal((rows, 1), 0.5, torch.float32, g).exp_().to(xt))  # rows of different sizes
        s["x"] = x
        s["weight"] = _normal((dim,), 0.2, torch.float32, g, mean=1.0).to(wt)
        s["bias"] = _normal((dim,), 0.2, torch.float32, g).to(wt)
        if case["step"]:
            s["dy"] = _normal((rows, dim), 1.0, TYPES[case["y"]], g)
    elif case["op"] == "linear":
        m, k, n, t = case["m"], case["k"], case["n"], TYPES[case["t"]]
        s["x"] = _normal((m, k), 1.0, t, g, pad=case["pad"])
        s["weight"] = _normal((n, k), k ** -0.5, t, g)
        s["bias"] = _normal((n,), 0.5, t, g) if case["bias"] else None
        s["residual"] = _normal((m, n), 1.0, t, g) if case["res"] else None
        if case["step"]:
            s["dy"] = _normal((m, n), 0.1, t, g)
    else:
        n, v, t = case["n"], case["v"], TYPES[case["t"]]
        z = _normal((n, v), 2.5, t, g, pad=case["pad"])
        s["targets"] = torch.randint(v, (n,), generator=g, device="cuda")
        if case["mask"] != "none":  # a third of the scores; with the type's lowest value never the token's own
            low = -math.inf if case["mask"] == "inf" else torch.finfo(t).min
            masked = torch.rand((n, v), generator=g, device="cuda") < 0.33
            if case["mask"] == "lowest":
                masked.scatter_(1, s["targets"][:, None], False)
            if n > 4:
                masked[3::61] = True  # rows that the mask leaves empty
            z.masked_fill_(masked, low)
        if n > 4:  # positions that have no token, as padding has none
            s["targets"][torch.rand(n, generator=g, device="cuda") < 0.05] = -1
        s["logits"] = z
        if case["step"]:
            s["dlogprob"] = _normal((n,), 1.0, torch.float32, g)
            s["dentropy"] = _normal((n,), 0.1, torch.float32, g)
    return s


# --- the plain forms ----------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain_ln(s):
    c, x, w, b = s["case"], s["x"].float(), s["weight"].float(), s["bias"].float()
    d = x - x.mean(1, keepdim=True)
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    xh = d * r
    out = {"y": (xh * w + b).to(TYPES[c["y"]])}
    if c["step"]:
        dy = s["dy"].float()
        g = dy * w
        out["dx"] = (r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))).to(s["x"].dtype)
        out["dweight"] = (dy * xh).sum(0).to(s["weight"].dtype)
        out["dbias"] = dy.sum(0).to(s["bias"].dtype)
    return out


def _plain_linear(s):
    c, x, w, t = s["case"], s["x"].float(), s["weight"].float(), s["x"].dtype
    z = x @ w.T
    if c["bias"]:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if c["res"]:
        y = y + s["residual"].float()
    out = {"y": y.to(t)}
    if c["step"]:
        p = s["dy"].float() * _act_slope(z, c["act"])
        out["dx"] = (p @ w).to(t)
        out["dweight"] = (p.T @ x).to(t)
        if c["bias"]:
            out["dbias"] = p.sum(0).to(t)
    return out


def _plain_logprobs(s):
    c, x, tg = s["case"], s["logits"].float(), s["targets"]
    n, v = x.shape
    top = x.amax(1, keepdim=True)
    none = top == -math.inf                       # rows with nothing to choose from
    d = (x - top.masked_fill(none, 0)) * c["scale"]
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    logs = torch.log(total)
    logp = (d - logs).masked_fill(none, -math.inf)
    p = (e / total).masked_fill(none, 0)
    entropy = -(p * logp.masked_fill(p == 0, 0)).sum(1)
    lp = logp.gather(1, tg.clamp(min=0)[:, None])[:, 0]
    out = {"logprob": torch.where(tg < 0, 0, lp), "entropy": entropy}
    if c["top"]:
        k = min(c["top"], v)
        bits = (x + 0.0).view(torch.int32).long()  # order of the values, then of the lowest index, in one number
        bits = torch.where(bits < 0, bits ^ 0x7FFF_FFFF, bits)
        key = (bits << 32) + (0x7FFF_FFFF - torch.arange(v, device=x.device))
        ids = key.topk(k, dim=1).indices
        tops = logp.gather(1, ids)
        ids = ids.masked_fill(x.gather(1, ids) == -math.inf, -1)
        more = (0, c["top"] - k)
        out["top_logprobs"] = torch.nn.functional.pad(tops, more, value=-math.inf)
        out["top_ids"] = torch.nn.functional.pad(ids, more, value=-1)
    if c["step"]:
        g, h = s["dlogprob"].masked_fill(tg < 0, 0)[:, None], s["dentropy"][:, None]
        dz = -p * (g + h * (logp.masked_fill(p == 0, 0) + entropy[:, None]))
        dz.scatter_add_(1, tg.clamp(min=0)[:, None], g)
        out["dlogits"] = (dz * c["scale"]).masked_fill(x == -math.inf, 0).to(s["logits"].dtype)
    return out


# --- the framework's operators -------------------------------------------------

def _own_ln(s):
    from paper_2504_01506_gb300 import dense

    c = s["case"]
    if not c["step"]:
        return {"y": dense.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, out_dtype=TYPES[c["y"]])}
    y, stats = dense.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, out_dtype=TYPES[c["y"]], save_stats=True)
    dx, dw, db = dense.layer_norm_backward(s["dy"], s["x"], s["weight"], stats)
    return {"y": y, "dx": dx, "dweight": dw, "dbias": db}


def _own_linear(s):
    from paper_2504_01506_gb300 import dense

    c = s["case"]
    if not c["step"]:
        return {"y": dense.linear(s["x"], s["weight"], s["bias"], activation=c["act"], residual=s["residual"])}
    y, pre = dense.linear(s["x"], s["weight"], s["bias"], activation=c["act"], residual=s["residual"], save_pre=True)
    dx, dw, db = dense.linear_backward(s["dy"], s["x"], s["weight"], pre, activation=c["act"], bias=c["bias"])
    out = {"y": y, "dx": dx, "dweight": dw}
    return {**out, "dbias": db} if c["bias"] else out


def _own_logprobs(s):
    from paper_2504_01506_gb300 import dense

    c = s["case"]
    r = dense.token_logprobs(s["logits"], s["targets"], top=c["top"], scale=c["scale"])
    out = {"logprob": r.logprob, "entropy": r.entropy}
    if c["top"]:
        out |= {"top_logprobs": r.top_logprobs, "top_ids": r.top_ids}
    if c["step"]:
        out["dlogits"] = dense.token_logprobs_backward(s["logits"], s["targets"], r, s["dlogprob"], s["dentropy"],
                                                       scale=c["scale"])
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return {"ln": _own_ln, "linear": _own_linear, "logprobs": _own_logprobs}[op](state)
    return {"ln": _plain_ln, "linear": _plain_linear, "logprobs": _plain_logprobs}[op](state)


# --- what a pass cannot do without ----------------------------------------------

def work(case):
    step = case["step"]
    if case["op"] == "ln":
        e, sx, sy = case["rows"] * case["dim"], SIZE[case["x"]], SIZE[case["y"]]
        params = 2 * case["dim"] * SIZE[case["w"]]
        return {"bytes": e * (sx + sy) * (2 if step else 1) + params * (2 if step else 1), "flops": e * (17 if step else 7)}
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        vals = m * k + n * k + m * n + (n if case["bias"] else 0) + (m * n if case["res"] else 0)
        if step:  # dy in; dx, dweight and dbias out
            vals += m * n + m * k + n * k + (n if case["bias"] else 0)
        return {"bytes": 2 * vals, "flops": 2 * m * n * k * (3 if step else 1)}
    n, e = case["n"], case["n"] * case["v"]
    return {"bytes": e * SIZE[case["t"]] * (2 if step else 1) + n * (16 + 12 * case["top"] + (8 if step else 0)),
            "flops": e * (13 if step else 6)}


# --- in 64 bits -------------------------------------------------------------------

def _exact_ln(s):
    x, w, b = s["x"].double(), s["weight"].double(), s["bias"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0)
    sd = (var + EPS).sqrt()
    out = {"y": torch.addcmul(b, (x - mean[:, None]) / sd[:, None], w)}
    if s["case"]["step"]:
        dy, dim = s["dy"].double(), x.shape[1]
        u = (x - mean[:, None]) / sd[:, None]
        along_u, along_1 = torch.einsum("rd,rd,d->r", dy, u, w), dy @ w
        out["dx"] = (dy * w - (along_1[:, None] + u * along_u[:, None]) / dim) / sd[:, None]
        out["dweight"], out["dbias"] = torch.einsum("rd,rd->d", dy, u), torch.einsum("rd->d", dy)
    return out


def _exact_linear(s):
    c, x, w = s["case"], s["x"].double(), s["weight"].double()
    z = torch.einsum("mk,nk->mn", x, w)
    if c["bias"]:
        z += s["bias"].double()
    if c["act"] == "relu":
        y, slope = torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0)
    elif c["act"] == "silu":
        q = torch.sigmoid(z)
        y, slope = z * q, q + z * q * torch.sigmoid(-z)
    elif c["act"] == "gelu_tanh":  # (1 + tanh u) / 2 = sigmoid(2 u)
        a = 2 * math.sqrt(2 / math.pi)
        q, r = torch.sigmoid(a * (z + 0.044715 * z ** 3)), torch.sigmoid(-a * (z + 0.044715 * z ** 3))
        y, slope = z * q, q + z * q * r * a * (1 + 0.134145 * z ** 2)
    else:
        y, slope = z, torch.ones_like(z)
    out = {"y": y + s["residual"].double() if c["res"] else y}
    if c["step"]:
        p = s["dy"].double() * slope
        out["dx"], out["dweight"] = torch.einsum("mn,nk->mk", p, w), torch.einsum("mn,mk->nk", p, x)
        if c["bias"]:
            out["dbias"] = torch.einsum("mn->n", p)
    return out


def _exact_logprobs(s):
    c, tg = s["case"], s["targets"]
    n, v = s["logits"].shape
    parts = []
    rows = max(1, (1 << 28) // v)
    for a in range(0, n, rows):
        z, t = s["logits"][a:a + rows].double() * c["scale"], tg[a:a + rows]
        z -= z.amax(1, keepdim=True).clamp(min=-1e300)  # (rows of nothing but the type's lowest value)
        lse = torch.logsumexp(z, 1)
        empty = (z == -math.inf).all(1)
        lp = z - lse[:, None]
        lp[empty] = -math.inf
        p = lp.exp()
        plogp = torch.special.entr(p)
        at = torch.arange(t.numel(), device=t.device)
        one = {"logprob": torch.where(t < 0, 0.0, lp[at, t.clamp(min=0)]), "entropy": plogp.sum(1)}
        if c["top"]:
            best = lp.sort(1, descending=True).values[:, :c["top"]] if v <= c["top"] else lp.topk(c["top"], 1).values
            full = torch.full((t.numel(), c["top"]), -math.inf, dtype=torch.float64, device=t.device)
            full[:, :best.shape[1]] = best
            one["top_logprobs"] = full
        if c["step"]:
            g = torch.where(t < 0, 0.0, s["dlogprob"][a:a + rows].double())
            h = s["dentropy"][a:a + rows].double()[:, None]
            dz = h * plogp - p * (h * one["entropy"][:, None] + g[:, None])
            dz[at, t.clamp(min=0)] += g
            dz[z == -math.inf] = 0
            one["dlogits"] = dz * c["scale"]
        parts.append(one)
    out = {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
    return {**out, "top_ids": None} if c["top"] else out


def exact(case, seed):
    s = prepare(case, seed)
    return {"ln": _exact_ln, "linear": _exact_linear, "logprobs": _exact_logprobs}[case["op"]](s)
