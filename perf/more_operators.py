"""More dense operators of a training step over the store, as they are measured.

Three operators, each alone: the gated block act(x Wg^T) * (x Wu^T) (with its backward pass), the cross entropy of a
linear layer over a large vocabulary that keeps no logits (with its gradients), and the AdamW step of many tensors
at once (states in 32 bits or in 8).  A "fwd" pass is serving's or scoring's; a "step" pass is a training step's
share of the operator: forward, then backward.

Widths and vocabularies are generic, or those that `perf/operators.py` takes for the products and the log
probabilities; the small networks are those of `examples/next_key.py`.

The plain form computes in 32 bits from elementary operations and rounds once at the end.  `exact` computes the
definitions in 64 bits.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2, "none": 0}
E4M3 = torch.float8_e4m3fn


def _gated(m, k, f, t, act, step, pad=0):
    return dict(op="gated", m=m, k=k, f=f, t=t, act=act, step=step, pad=pad)


def _xent(n, k, v, t, step, scale=1.0, pad=0):
    return dict(op="xent", n=n, k=k, v=v, t=t, step=step, scale=scale, pad=pad)


def _adamw(net, count, size, p, g, copy, bits, t, clip=False):
    """net: "block" (`count` times two size x 3 size matrices, one the other way round and two vectors), "tower" (`count` layers
    of size x size with their biases) or "mixed" (`count` tensors of 1 to `size` values)."""
    return dict(op="adamw", net=net, count=count, size=size, p=p, g=g, copy=copy, bits=bits, t=t, clip=clip)


def listed():
    return [
        # A single generated token through a wide gated block: two weights are read once, nothing else counts.
        dict(name="gated_token", **_gated(1, 4_096, 12_288, "bf16", "silu", False)),
        # A small serving batch.
        dict(name="gated_serve", **_gated(26, 1_024, 4_096, "fp16", "gelu_tanh", False)),
        # Training an odd network on an odd batch: no row starts on a 16-byte boundary.
        dict(name="gated_odd_step", **_gated(4_099, 777, 1_001, "bf16", "silu", True)),
        # Training a wide block: the largest.
        dict(name="gated_wide_step", **_gated(8_192, 4_096, 12_288, "bf16", "silu", True)),
        # Scoring 16 samples over relation-sized classes: latency.
        dict(name="xent_score", **_xent(16, 128, 15_000, "fp16", False)),
        # Scoring one token of a large vocabulary: the weight is read once.
        dict(name="xent_token", **_xent(1, 2_048, 131_072, "bf16", False)),
        # Training over an odd vocabulary, with a temperature; rows off 16 bytes.
        dict(name="xent_odd_step", **_xent(2_051, 777, 50_001, "bf16", True, scale=1.25)),
        # Training over a large vocabulary: the largest.
        dict(name="xent_wide_step", **_xent(8_192, 2_048, 131_072, "bf16", True)),
        # The step of a small tower over the store's rows: latency.
        dict(name="adamw_tower", **_adamw("tower", 4, 256, "fp32", "bf16", "bf16", 32, 100)),
        # Tensors of every size, odd ones, one value among them; gradients clipped by a factor on the device.
        dict(name="adamw_mixed", **_adamw("mixed", 120, 3_000_000, "fp32", "fp16", "none", 8, 1, clip=True)),
        # A wide network, 32-bit states, 16-bit copies of the weights for the products.
        dict(name="adamw_wide", **_adamw("block", 3, 4_096, "fp32", "bf16", "bf16", 32, 1_000)),
        # The same with 8-bit states.
        dict(name="adamw_wide_8bit", **_adamw("block", 3, 4_096, "fp32", "bf16", "bf16", 8, 1_000)),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def _width(rng, lo, hi):
    """As _spread; mostly a multiple of 8, as widths are, else any."""
    v = _spread(rng, lo, hi)
    return v if rng.random() < 0.35 else max(lo, v // 8 * 8)


def draw(rng):
    """Gated blocks of 1 to 16,384 rows over widths 16 to 12,288; 1 to 16,384 rows of width 16 to 4,096 over 2 to 262,144
    tokens; networks of 1 to 200 tensors and up to 450 million weights: every type, direction, activation and kind of
    state, contiguous rows and slices of wider ones."""
    op = rng.choice(["gated", "gated", "xent", "xent", "adamw"])
    step = rng.random() < 0.6
    pad = rng.choice([0, 0, 0, 8, 5])
    t = rng.choice(["bf16", "bf16", "fp16"])
    if op == "gated":
        k, f = _width(rng, 16, 8_192), _width(rng, 16, 12_288)
        m = _spread(rng, 1, min(16_384, 8_192 * 4_096 * 12_288 // (f * k)))
        return _gated(m, k, f, t, rng.choice(["none", "relu", "gelu_tanh", "silu", "silu"]), step, pad)
    if op == "xent":
        k = _width(rng, 16, 4_096)
        v = _spread(rng, 2, 262_144) if rng.random() < 0.4 else _width(rng, 256, 262_144)
        n = _spread(rng, 1, min(16_384, 8_192 * 2_048 * 131_072 // (k * v), 8_192 * 131_072 // v))
        return _xent(n, k, v, t, step, rng.choice([1.0, 1.0, 0.7, 1.25]), pad)
    p = rng.choice(["fp32", "fp32", "bf16", "fp16"])
    g = rng.choice(["fp32", "bf16", "fp16"]) if p == "fp32" else p
    copy = rng.choice(["none", "bf16", "fp16"]) if p == "fp32" else "none"
    bits, when, clip = rng.choice([32, 8]), rng.choice([1, 2, 37, 5_000]), rng.random() < 0.5
    net = rng.choice(["block", "tower", "mixed"])
    if net == "mixed":
        return _adamw(net, rng.randint(1, 200), _spread(rng, 1, 4_000_000), p, g, copy, bits, when, clip)
    size = _width(rng, 16, 4_096)
    return _adamw(net, rng.randint(1, min(8, 3 * 4_096 ** 2 // size ** 2)), size, p, g, copy, bits, when, clip)


# --- inputs -----------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator("cuda")
    g.manual_seed((seed * 1_000_003 + stream * 7_919 + 29) & 0x7FFF_FFFF_FFFF)
    return g


def _normal(shape, sigma, dtype, gen, mean=0.0, pad=0):
    """N(mean, sigma) values; with `pad`, rows that are slices of rows `pad` values wider."""
    full = (*shape[:-1], shape[-1] + pad)
    x = torch.empty(full, device="cuda", dtype=dtype).normal_(mean, sigma, generator=gen)
    return x[..., :shape[-1]] if pad else x


def _shapes(case):
    n, s = case["count"], case["size"]
    if case["net"] == "block":
        return [q for _ in range(n) for q in ((3 * s, s), (3 * s, s), (s, 3 * s), (s,), (s,))]
    if case["net"] == "tower":
        return [q for _ in range(n) for q in ((s, s), (s,))]
    # from 1 to s values, evenly over the logarithm, odd more often than not
    return [(max(1, int(s ** (i / max(1, n - 1))) - i % 2),) for i in range(n)]


def _views(s, name, shapes, dtype):
    """One buffer (zeros) for all of a network's tensors, each from a multiple of 128 values on; s[name]: the tensors."""
    at, places = 0, []
    for q in shapes:
        places.append(at)
        at += (math.prod(q) + 127) // 128 * 128
    flat = torch.zeros(at, device="cuda", dtype=dtype)
    s[name] = [flat[a:a + math.prod(q)].view(q) for a, q in zip(places, shapes)]
    return flat


def prepare(case, seed):
    g = _gen(seed, 1)
    s = {"case": case}
    if case["op"] == "gated":
        m, k, f, t = case["m"], case["k"], case["f"], TYPES[case["t"]]
        s["x"] = _normal((m, k), 1.0, t, g, pad=case["pad"])
        s["w_gate"] = _normal((f, k), k ** -0.5, t, g)
        s["w_up"] = _normal((f, k), k ** -0.5, t, g)
        if case["step"]:
            s["dh"] = _normal((m, f), 0.1, t, g, pad=case["pad"])
    elif case["op"] == "xent":
        n, k, v, t = case["n"], case["k"], case["v"], TYPES[case["t"]]
        s["x"] = _normal((n, k), 1.0, t, g, pad=case["pad"])
        s["weight"] = _normal((v, k), 2.0 * k ** -0.5, t, g)
        s["targets"] = torch.randint(v, (n,), generator=g, device="cuda")
        if n > 4:  # positions that have no token, as padding has none
            s["targets"][torch.rand(n, generator=g, device="cuda") < 0.05] = -1
        if case["step"]:  # a mean over the tokens, these weighted; in fp16 the loss is scaled, so that gradients do not vanish
            s["dloss"] = (torch.rand(n, generator=g, device="cuda") + 0.5) * ((4_096.0 if case["t"] == "fp16" else 1.0) / n)
    else:
        pt, gt, bits = TYPES[case["p"]], TYPES[case["g"]], case["bits"]
        shapes, first, state = _shapes(case), case["t"] == 1, torch.float32 if bits == 32 else E4M3
        blocks = [(2, (math.prod(q) + 255) // 256) for q in shapes]
        s["flat"] = {"params": _views(s, "params", shapes, pt), "m": _views(s, "m", shapes, state), "v": _views(s, "v", shapes, state)}
        if case["copy"] != "none":
            s["flat"]["copies"] = _views(s, "copies", shapes, TYPES[case["copy"]])
        if bits == 8:
            s["flat"]["scales"] = _views(s, "scales", blocks, torch.float32)
        s["grads"] = []
        for i, shape in enumerate(shapes):
            wide = shape[-1] ** -0.5 if len(shape) > 1 else 0.1
            s["params"][i].normal_(0, wide, generator=g)
            s["grads"].append(_normal(shape, 1e-3, gt, g))
            if case["copy"] != "none":
                s["copies"][i].copy_(s["params"][i])
            if first:
                continue
            m, r = _normal(shape, 3e-4, torch.float32, g), _normal(shape, 2e-4, torch.float32, g, mean=1e-3).abs_()
            if bits == 32:
                s["m"][i].copy_(m)
                s["v"][i].copy_(r.mul_(r))
            else:  # at a scale of 2^-16: codes of up to 448
                s["scales"][i].fill_(2.0 ** -16)
                s["m"][i].copy_(m.mul_(2.0 ** 16).clamp_(-448, 448).to(E4M3))
                s["v"][i].copy_(r.mul_(2.0 ** 16).clamp_(max=448).to(E4M3))
        s["clip"] = torch.tensor([0.37], device="cuda") if case["clip"] else None
        s["seed"] = (seed * 2_654_435_761 + 12_345) & 0xFFFF_FFFF
    return s


HYPER = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)


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


def _plain_gated(s):
    c, t = s["case"], s["x"].dtype
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    gate, up = x @ wg.T, x @ wu.T
    a = _act(gate, c["act"])
    out = {"h": (a * up).to(t)}
    if c["step"]:
        dh = s["dh"].float()
        du = dh * a
        dg = dh * up * _act_slope(gate, c["act"])
        out["dx"] = (dg @ wg + du @ wu).to(t)
        out["dw_gate"] = (dg.T @ x).to(t)
        out["dw_up"] = (du.T @ x).to(t)
    return out


def _plain_xent(s):
    c, tg, t = s["case"], s["targets"], s["x"].dtype
    x, w = s["x"].float(), s["weight"].float()
    z = (x @ w.T) * c["scale"]
    top = z.amax(1, keepdim=True)
    z -= top
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    at = tg.clamp(min=0)[:, None]
    loss = (torch.log(total) - z.gather(1, at))[:, 0].masked_fill(tg < 0, 0)
    out = {"loss": loss}
    if c["step"]:
        del z
        g = s["dloss"].masked_fill(tg < 0, 0)[:, None] * c["scale"]
        p = e.mul_(g / total)
        p.scatter_add_(1, at, -g)
        out["dx"] = (p @ w).to(t)
        out["dweight"] = (p.T @ x).to(t)
    return out


MASK = 0xFFFF_FFFF


def _mix(h):
    """A hash of 32 bits (whole numbers, or tensors of them)."""
    h = h ^ (h >> 16)
    h = (h * 0x6A09E667) & MASK
    h = h ^ (h >> 15)
    h = (h * 0xBB67AE85) & MASK
    return h ^ (h >> 16)


def _dither(key, n):
    """Two numbers from -0.5 up to 0.5 for each of n values."""
    h = (torch.arange(n, device="cuda") * 0x9E3779B9 + key) & MASK
    h = h ^ (h >> 15)
    unit = lambda a: ((a >> 9) | 0x3F800000).int().view(torch.float32) - 1.5  # noqa: E731
    return unit((h * 0x6A09E667) & MASK), unit((h * 0xBB67AE85) & MASK)


def _to_codes(x, dither):
    """(e4m3 codes of x in blocks of 256 values, the blocks' scales): the least power of two that brings a block's
    largest value to 448 or less; rounded up or down by chance, so that the mean is x."""
    n = x.numel()
    blocks = (n + 255) // 256
    b = torch.nn.functional.pad(x, (0, blocks * 256 - n)).view(blocks, 256)
    most = b.abs().amax(1).view(torch.int32)
    power = (most >> 23) - 8 + ((most & 0x7FFFFF) > 0x600000).int()
    scale = (power.clamp(min=1) << 23).view(torch.float32)
    q = x * (1 / scale).repeat_interleave(256)[:n]
    step = ((q.view(torch.int32) & 0x7F800000).clamp(min=(127 - 6) << 23)).view(torch.float32) * 0.125
    return (q + step * dither).clamp(-448, 448), scale


def _plain_adamw_one(s, i):
    c, p, m, v = s["case"], s["params"][i], s["m"][i], s["v"][i]
    (b1, b2), t = HYPER["betas"], c["t"]
    n = p.numel()
    g = s["grads"][i].float().view(-1)
    if s["clip"] is not None:
        g = g * s["clip"]
    if c["bits"] == 32:
        m0, v0 = m.view(-1), v.view(-1)
    else:
        sm, sr = s["scales"][i].repeat_interleave(256, dim=1)[:, :n]
        m0, r0 = m.float().view(-1) * sm, v.float().view(-1) * sr
        v0 = r0 * r0
    m1 = m0 * b1 + g * (1 - b1)
    v1 = v0 * b2 + (g * g) * (1 - b2)
    r1 = torch.sqrt(v1)
    x = p.float().view(-1)
    x = x * (1 - HYPER["lr"] * HYPER["weight_decay"]) - HYPER["lr"] / (1 - b1 ** t) * m1 / (r1 / math.sqrt(1 - b2 ** t) + HYPER["eps"])
    p.copy_(x.view(p.shape))
    if "copies" in s:
        s["copies"][i].copy_(x.view(p.shape))
    if c["bits"] == 32:
        m.copy_(m1.view(m.shape))
        v.copy_(v1.view(v.shape))
        return
    key = _mix((_mix((_mix(s["seed"]) + t) & MASK) + i) & MASK)
    dm, dr = _dither(key, n)
    q, sm = _to_codes(m1, dm)
    m.copy_(q.view(m.shape).to(E4M3))
    q, sr = _to_codes(r1, dr)
    q = torch.where(r1 > 0, q.clamp(min=2.0 ** -9), 0.0)  # (what is not 0 stays so: it divides)
    v.copy_(q.view(v.shape).to(E4M3))
    s["scales"][i].copy_(torch.stack([sm, sr]))


def _plain_adamw(s):
    for i in range(len(s["params"])):
        _plain_adamw_one(s, i)
    return dict(s["flat"])


# --- the framework's operators -------------------------------------------------

def _own_gated(s):
    from paper_2504_01506_gb300 import dense

    c = s["case"]
    if not c["step"]:
        return {"h": dense.gated_linear(s["x"], s["w_gate"], s["w_up"], activation=c["act"])}
    h, gate, up = dense.gated_linear(s["x"], s["w_gate"], s["w_up"], activation=c["act"], save_pre=True)
    dx, dwg, dwu = dense.gated_linear_backward(s["dh"], s["x"], s["w_gate"], s["w_up"], gate, up, activation=c["act"])
    return {"h": h, "dx": dx, "dw_gate": dwg, "dw_up": dwu}


def _own_xent(s):
    from paper_2504_01506_gb300 import dense

    c = s["case"]
    r = dense.linear_cross_entropy(s["x"], s["weight"], s["targets"], scale=c["scale"])
    if not c["step"]:
        return {"loss": r.loss}
    dx, dw = dense.linear_cross_entropy_backward(s["dloss"], s["x"], s["weight"], s["targets"], r, scale=c["scale"])
    return {"loss": r.loss, "dx": dx, "dweight": dw}


def _own_adamw(s):
    from paper_2504_01506_gb300 import dense

    state = dense.AdamWState(s["m"], s["v"], s.get("scales"))
    dense.adamw(s["params"], s["grads"], state, s["case"]["t"], **HYPER, grad_scale=s["clip"], copies=s.get("copies"), seed=s["seed"])
    return dict(s["flat"])


def run(state):
    op = state["case"]["op"]
    if own:
        return {"gated": _own_gated, "xent": _own_xent, "adamw": _own_adamw}[op](state)
    return {"gated": _plain_gated, "xent": _plain_xent, "adamw": _plain_adamw}[op](state)


# --- what a pass cannot do without ----------------------------------------------

def work(case):
    if case["op"] == "gated":
        m, k, f, step = case["m"], case["k"], case["f"], case["step"]
        vals = m * k + 2 * f * k + m * f
        if step:  # dh in; dx and the weights' gradients out
            vals += m * f + m * k + 2 * f * k
        return {"bytes": 2 * vals, "flops": 4 * m * k * f * (3 if step else 1)}
    if case["op"] == "xent":  # without logits that are kept, the backward pass has them to compute again
        n, k, v, step = case["n"], case["k"], case["v"], case["step"]
        return {"bytes": 2 * (n * k + v * k) * (2 if step else 1) + n * (16 if step else 12), "flops": 2 * n * k * v * (4 if step else 1)}
    n = sum(math.prod(q) for q in _shapes(case))
    state = 16 if case["bits"] == 32 else 4
    return {"bytes": n * (2 * SIZE[case["p"]] + SIZE[case["g"]] + state + SIZE[case["copy"]]), "flops": 16 * n}


# --- in 64 bits -------------------------------------------------------------------

def _exact_gated(s):
    c, x, wg, wu = s["case"], s["x"].double(), s["w_gate"].double(), s["w_up"].double()
    z, u = torch.einsum("mk,fk->mf", x, wg), torch.einsum("mk,fk->mf", x, wu)
    if c["act"] == "relu":
        a, slope = torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0).double()
    elif c["act"] == "silu":
        q = torch.sigmoid(z)
        a, slope = z * q, q + z * q * torch.sigmoid(-z)
    elif c["act"] == "gelu_tanh":  # (1 + tanh u) / 2 = sigmoid(2 u)
        b = 2 * math.sqrt(2 / math.pi)
        q, r = torch.sigmoid(b * (z + 0.044715 * z ** 3)), torch.sigmoid(-b * (z + 0.044715 * z ** 3))
        a, slope = z * q, q + z * q * r * b * (1 + 0.134145 * z ** 2)
    else:
        a, slope = z, torch.ones_like(z)
    out = {"h": a * u}
    if c["step"]:
        dh = s["dh"].double()
        dg, du = dh * u * slope, dh * a
        out["dx"] = torch.einsum("mf,fk->mk", dg, wg) + torch.einsum("mf,fk->mk", du, wu)
        out["dw_gate"], out["dw_up"] = torch.einsum("mf,mk->fk", dg, x), torch.einsum("mf,mk->fk", du, x)
    return out


def _exact_xent(s):
    c, tg, x, w = s["case"], s["targets"], s["x"].double(), s["weight"].double()
    n, v = x.shape[0], w.shape[0]
    loss, dx, dw = [], [], torch.zeros_like(w) if c["step"] else None
    rows = max(1, (1 << 28) // v)
    for a in range(0, n, rows):
        t, y = tg[a:a + rows], x[a:a + rows]
        z = torch.einsum("nk,vk->nv", y, w) * c["scale"]
        lse = torch.logsumexp(z, 1)
        at = torch.arange(t.numel(), device=t.device)
        loss.append(torch.where(t < 0, 0.0, lse - z[at, t.clamp(min=0)]))
        if c["step"]:
            g = torch.where(t < 0, 0.0, s["dloss"][a:a + rows].double()) * c["scale"]
            p = torch.softmax(z, 1) * g[:, None]
            p[at, t.clamp(min=0)] -= g
            dx.append(p @ w)
            dw += p.T @ y
    out = {"loss": torch.cat(loss)}
    return {**out, "dx": torch.cat(dx), "dweight": dw} if c["step"] else out


def _exact_adamw(s):
    c, t, (b1, b2) = s["case"], s["case"]["t"], HYPER["betas"]
    wide, shapes = {}, _shapes(c)
    out = {"params": _views(wide, "params", shapes, torch.float64), "m": None, "v": None}  # (codes are rounded by chance, and have no such value)
    if c["bits"] == 32:
        out["m"], out["v"] = _views(wide, "m", shapes, torch.float64), _views(wide, "v", shapes, torch.float64)
    if "copies" in s:
        out["copies"] = out["params"]
    if c["bits"] == 8:
        out["scales"] = None
    for i, p in enumerate(s["params"]):
        g = s["grads"][i].double()
        if s["clip"] is not None:
            g = g * s["clip"].double()
        m, v = s["m"][i].double(), s["v"][i].double()
        if c["bits"] == 8:
            sm, sr = s["scales"][i].double().repeat_interleave(256, dim=1)[:, :p.numel()]
            m, v = m * sm.view(m.shape), (v * sr.view(v.shape)) ** 2
        m, v = torch.lerp(g, m, b1), torch.lerp(g ** 2, v, b2)
        root = (v / (1 - b2 ** t)).sqrt()
        x = p.double()
        wide["params"][i].copy_(x - HYPER["lr"] * (HYPER["weight_decay"] * x + m / (1 - b1 ** t) / (root + HYPER["eps"])))
        if c["bits"] == 32:
            wide["m"][i].copy_(m)
            wide["v"][i].copy_(v)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"gated": _exact_gated, "xent": _exact_xent, "adamw": _exact_adamw}[case["op"]](s)
